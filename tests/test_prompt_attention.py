"""Causal attention of packed prompts, against softmax attention in 64 bits; refusals; and prompts, pages and decode steps together."""
import math

import numpy as np
import pytest
import torch

import paper_2604_16734_amd as K
from kvp_workload import Segment
from tests.test_paged_decode import check, reference
from tests.test_pages import DEV, P16, P4, Pool, gpu, int32, laid_out


def causal(q, k, v, begin, scale, heads=None):
    """(out, size, most) as in test_paged_decode.reference, in 64 bits on the GPU; rows of no prompt are NaN.  What a row does not see is left
    out, not multiplied by zero."""
    q, k, v = (x.to(DEV).double() for x in (q, k, v))
    n, hq, d = q.shape
    group, out, size, most = hq // k.shape[1], torch.full_like(q, float("nan")), torch.full_like(q, float("nan")), 0.0
    for s in range(len(begin) - 1):
        at = slice(begin[s], begin[s + 1])
        m = begin[s + 1] - begin[s]
        if m <= 0:
            continue
        unseen = torch.ones(m, m, dtype=torch.bool, device=DEV).triu(1)
        for h in range(hq) if heads is None else heads:
            kh, vh = k[at, h // group], v[at, h // group]
            logits = (q[at, h] @ kh.T * scale).masked_fill(unseen, -math.inf)
            most = max(most, float((q[at, h].abs() @ torch.nan_to_num(kh, posinf=0, neginf=0).abs().T).max()) * scale)
            w = torch.softmax(logits, -1)
            if torch.isfinite(vh).all():
                out[at, h], size[at, h] = w @ vh, w @ vh.abs()
            else:
                for i in range(m):
                    out[begin[s] + i, h] = w[i, :i + 1] @ vh[:i + 1]
                    size[begin[s] + i, h] = w[i, :i + 1] @ vh[:i + 1].abs()
    return out.cpu().numpy(), size.cpu().numpy(), most


def same(out, ref, size, most, d):
    rows = np.isfinite(ref).all(axis=-1)
    check(out.cpu()[torch.from_numpy(rows)], ref[rows], size[rows], most, d)


def randn(gen, *shape, scale=1.0):
    return (scale * torch.randn(shape, generator=gen)).to(torch.bfloat16)


HEADS = [(4, 4, 64), (32, 8, 128), (7, 1, 128), (16, 4, 64), (28, 4, 128), (3, 3, 128), (8, 1, 64)]
LENGTHS = [[1], [2, 0, 31, 32, 33], [63, 64, 65], [127, 128, 129, 1], [191, 200, 256, 257], [608], [0, 0, 5, 0], [1000, 17, 0, 333]]


@gpu
@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_against_64_bits(hq, hkv, d, lengths):
    gen = torch.Generator().manual_seed(hq + d + sum(lengths))
    before, behind = (3, 5) if len(lengths) > 1 else (0, 0)
    begin = (np.concatenate([[0], np.cumsum(lengths)]) + before).tolist()
    n = begin[-1] + behind
    q, k, v = randn(gen, n, hq, d, scale=1.5), randn(gen, n, hkv, d), randn(gen, n, hkv, d)
    k[:before], v[:before], k[begin[-1]:], v[begin[-1]:] = (float("nan"),) * 4
    out = torch.full((n, hq, d), 7.0, dtype=torch.bfloat16, device=DEV)
    print("prompt attention", hq, hkv, d, lengths, flush=True)
    K.prompt_attention(q.to(DEV), k.to(DEV), v.to(DEV), int32(begin), out=out)
    torch.cuda.synchronize()
    ref, size, most = causal(q, k, v, begin, d ** -0.5)
    same(out, ref, size, most, d)
    assert (out[:before] == 7).all() and (out[begin[-1]:] == 7).all()


@gpu
@pytest.mark.parametrize("hq,hkv,d,n", [(8, 2, 128, 4097), (2, 1, 64, 5000), (1, 1, 128, 9001), (24, 8, 64, 2900), (20, 4, 128, 3500)])
def test_long_prompts(hq, hkv, d, n):
    gen = torch.Generator().manual_seed(n)
    q, k, v = randn(gen, n, hq, d, scale=2.0), randn(gen, n, hkv, d), randn(gen, n, hkv, d)
    out = K.prompt_attention(q.to(DEV), k.to(DEV), v.to(DEV), int32([0, n]), softmax_scale=0.2)
    torch.cuda.synchronize()
    ref, size, most = causal(q, k, v, [0, n], 0.2)
    same(out, ref, size, most, d)


@gpu
@pytest.mark.parametrize("how,other", [("rows", "heads"), ("heads", "projection"), ("projection", "rows")])
@pytest.mark.parametrize("hq,hkv,d", [(6, 2, 128), (16, 8, 64), (84, 28, 128), (96, 6, 64)])
def test_strides(hq, hkv, d, how, other):
    gen = torch.Generator().manual_seed(d)
    begin = [0, 70, 333]
    q, k, v = randn(gen, 333, hq, d), randn(gen, 333, hkv, d), randn(gen, 333, hkv, d)
    (qd, _), (kd, _), (vd, _) = laid_out(q, how), laid_out(k, other), laid_out(v, how)
    out, room = laid_out(torch.full_like(q, 3.0), other)
    K.prompt_attention(qd, kd, vd, int32(begin), out=out)
    plain = K.prompt_attention(q.to(DEV), k.to(DEV), v.to(DEV), int32(begin))
    torch.cuda.synchronize()
    assert torch.equal(out, plain)
    if room is not None:
        assert int((room == 7.0).sum()) >= room.numel() - q.numel()
    ref, size, most = causal(q, k, v, begin, d ** -0.5)
    same(out, ref, size, most, d)


@gpu
@pytest.mark.parametrize("hq,lengths", [(4, [640, 60]), (48, [700]), (96, [640, 60]), (28, [16] * 43 + [12])])
def test_rows_beyond_32_bits(hq, lengths):
    """Rows 8 MiB apart: in every tensor the last ones lie 5.7 GB behind the first."""
    gen = torch.Generator().manual_seed(hq)
    n, hkv, d, far = sum(lengths), 2, 128, 1 << 22
    begin = int32(np.concatenate([[0], np.cumsum(lengths)]).tolist())
    q, k, v = (x.to(DEV) for x in (randn(gen, n, hq, d), randn(gen, n, hkv, d), randn(gen, n, hkv, d)))
    plain = K.prompt_attention(q, k, v, begin)
    room = torch.empty(n * far, dtype=torch.bfloat16, device=DEV)
    at = 0
    views = []
    for x in (q, k, v, plain):
        views.append(room.as_strided(x.shape, (far, d, 1), at))
        at += x.shape[1] * d
    for view, x in zip(views, (q, k, v)):
        view.copy_(x)
    K.prompt_attention(*views[:3], begin, out=views[3])
    torch.cuda.synchronize()
    assert torch.equal(views[3], plain)


@gpu
def test_many_prompts():
    gen = torch.Generator().manual_seed(2)
    lengths = [0] * 70 + [int(x) for x in torch.randint(0, 300, (90,), generator=gen)] + [0] * 40
    begin = np.concatenate([[0], np.cumsum(lengths)]).tolist()
    n = begin[-1]
    q, k, v = randn(gen, n, 4, 64), randn(gen, n, 2, 64), randn(gen, n, 2, 64)
    out = K.prompt_attention(q.to(DEV), k.to(DEV), v.to(DEV), int32(begin))
    torch.cuda.synchronize()
    ref, size, most = causal(q, k, v, begin, 0.125)
    assert np.isfinite(ref).all()
    same(out, ref, size, most, 64)


@gpu
@pytest.mark.parametrize("how", ["rows", "projection"])
@pytest.mark.parametrize("hq,hkv,d", [(16, 4, 128), (28, 4, 64), (32, 32, 128), (20, 20, 64)])
def test_short_prompts(hq, hkv, d, how):
    """Many of a few rows and one longer one; rows around them with NaNs, large logits, first keys that weigh nothing, and values that only the last
    row of a prompt sees."""
    gen = torch.Generator().manual_seed(hq + d)
    lengths = [0, 1, 2, 31, 32, 33, 63, 64, 65, 300, 0] + [int(x) for x in torch.randint(1, 60, (40,), generator=gen)] + [17]
    begin = (np.concatenate([[0], np.cumsum(lengths)]) + 2).tolist()
    n = begin[-1] + 3
    q, k, v = randn(gen, n, hq, d, scale=1.5), randn(gen, n, hkv, d), randn(gen, n, hkv, d)
    q[begin[20]:begin[24]] *= 32
    k[begin[9]:begin[9] + 40] = -math.inf
    q[begin[9]:begin[10]] = q[begin[9]:begin[10]].abs() + 0.125
    k[begin[9] + 40:begin[10]] = -k[begin[9] + 40:begin[10]].abs() - 0.5
    last = [begin[i + 1] - 1 for i in range(12, len(lengths))]
    v[last] = math.inf
    k[:2], v[:2], k[begin[-1]:], v[begin[-1]:] = (float("nan"),) * 4
    (qd, _), (kd, _), (vd, _) = (laid_out(x, how) for x in (q, k, v))
    out, room = laid_out(torch.full_like(q, 7.0), how)
    print("short prompts", hq, hkv, d, how, flush=True)
    K.prompt_attention(qd, kd, vd, int32(begin), out=out)
    torch.cuda.synchronize()
    clean = v.clone()
    clean[last] = 0.0
    ref, size, most = causal(q, k, clean, begin, d ** -0.5)
    ref[last], ref[begin[9]:begin[9] + 40] = math.nan, math.nan
    assert np.isfinite(ref).all(axis=(1, 2)).sum() == sum(lengths) - len(last) - 40
    same(out, ref, size, most, d)
    assert not torch.isfinite(out[last]).any()
    assert (out[:2] == 7).all() and (out[begin[-1]:] == 7).all()


# few rows for the chip, many, and many of few heads
@gpu
@pytest.mark.parametrize("n,hq,hkv", [(450, 4, 2), (450, 96, 48), (900, 24, 12)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("what", [float("inf"), float("nan"), -3e38])
def test_what_a_row_does_not_see_has_no_part_in_it(d, what, n, hq, hkv):
    """Keys and values that are not finite, or as small as their type has them: rows before them have the bits that they have without them."""
    gen = torch.Generator().manual_seed(d)
    q, k, v = (x.to(DEV) for x in (randn(gen, n, hq, d), randn(gen, n, hkv, d), randn(gen, n, hkv, d)))
    begin = int32([0, 100, n])
    good = K.prompt_attention(q, k, v, begin)
    for row in (100, 141, 200, 317, n - 1):
        k2, v2 = k.clone(), v.clone()
        k2[row, 0, 3], v2[row, 0, 5] = what, what
        out = K.prompt_attention(q, k2, v2, begin)
        torch.cuda.synchronize()
        clean = torch.ones(n, hq, dtype=torch.bool, device=DEV)
        clean[row:, :2] = False
        tol = good.abs() * 2.0 ** -7 + 2.0 ** -8 * v.abs().max()         # two roundings of results, and of weights, which the slow way does not round
        assert ((out - good).abs() <= tol)[clean].all() and torch.isfinite(out[clean]).all()
        if what == what and what > 0:
            ref = K.prompt_attention(q, k, v2, begin)
            torch.cuda.synchronize()
            assert torch.isinf(ref[row:, :2, 5]).all() and torch.isfinite(ref[row:, :2, 6]).all()


@gpu
@pytest.mark.parametrize("hq,hkv", [(2, 1), (96, 48), (48, 24)])
@pytest.mark.parametrize("d", [64, 128])
def test_logits_that_run_away(d, hq, hkv):
    """Logits far above those of the first keys, past what a fixed reference takes, in single rows and in all of them."""
    gen = torch.Generator().manual_seed(7)
    n = 400
    for rows in (slice(250, 251), slice(40, n)):
        q, k, v = randn(gen, n, hq, d), randn(gen, n, hkv, d), randn(gen, n, hkv, d)
        q[rows] = (30 * q[rows].float()).to(torch.bfloat16)
        k[200] = q[250, 0]
        k[300:] = (10 * k[300:].float()).to(torch.bfloat16)
        out = K.prompt_attention(q.to(DEV), k.to(DEV), v.to(DEV), int32([0, n]))
        torch.cuda.synchronize()
        ref, size, most = causal(q, k, v, [0, n], d ** -0.5)
        same(out, ref, size, most, d)


# one prompt whose rows two groups of waves share: tiles of 64 keys in turns, each group with a reference of its own
TWO_GROUPS = [(48, 24, 500), (24, 12, 900)]


@gpu
@pytest.mark.parametrize("hq,hkv,n", TWO_GROUPS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("top", [60, 100, 127, 200])
@pytest.mark.parametrize("first,late", [(0, 100), (64, 140), (0, 239), (64, 300)])
def test_references_of_two_groups_far_apart(d, hq, hkv, n, top, first, late):
    """The first keys of one group lie 2^top above those of the other, which has a key of nearly that weight later on.  Logits are in powers
    of two, in channel 0."""
    gen = torch.Generator().manual_seed(n + top)
    q, k, v = randn(gen, n, hq, d, scale=0.25), randn(gen, n, hkv, d, scale=0.25), randn(gen, n, hkv, d)
    q[..., 0], k[..., 0] = 1.0, 0.0
    k[first, :, 0], k[late, :, 0] = float(top), top - 0.5
    v[first], v[late] = v[first] - 2.0, v[late] + 2.0
    scale = math.log(2)
    out = K.prompt_attention(q.to(DEV), k.to(DEV), v.to(DEV), int32([0, n]), softmax_scale=scale)
    torch.cuda.synchronize()
    ref, size, most = causal(q, k, v, [0, n], scale)
    same(out, ref, size, most, d)


@gpu
@pytest.mark.parametrize("hq,hkv,n", TWO_GROUPS)
@pytest.mark.parametrize("d", [64, 128])
def test_logits_that_run_away_in_two_groups(d, hq, hkv, n):
    gen = torch.Generator().manual_seed(n + d)
    for rows in (slice(250, 251), slice(40, n)):
        q, k, v = randn(gen, n, hq, d), randn(gen, n, hkv, d), randn(gen, n, hkv, d)
        q[rows] = (30 * q[rows].float()).to(torch.bfloat16)
        k[200] = q[250, 0]
        k[300:] = (10 * k[300:].float()).to(torch.bfloat16)
        out = K.prompt_attention(q.to(DEV), k.to(DEV), v.to(DEV), int32([0, n]))
        torch.cuda.synchronize()
        ref, size, most = causal(q, k, v, [0, n], d ** -0.5)
        same(out, ref, size, most, d)


@gpu
@pytest.mark.parametrize("hq,hkv", [(2, 1), (96, 48), (48, 24)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", [0.25, 20.0])
def test_first_keys_that_weigh_nothing(d, hq, hkv, size):
    """Logits of minus infinity before all others, which are about 0 or far below it."""
    gen = torch.Generator().manual_seed(8)
    n, first = 500, 40
    q, k, v = randn(gen, n, hq, d).abs() + 0.125, -size * (1 + randn(gen, n, hkv, d).abs()), randn(gen, n, hkv, d)
    k[:first] = -math.inf
    out = K.prompt_attention(q.to(DEV), k.to(DEV), v.to(DEV), int32([0, n]))
    torch.cuda.synchronize()
    ref, size, most = causal(q, k, v, [0, n], d ** -0.5)
    assert np.isfinite(ref[first:]).all()
    same(out, ref, size, most, d)


@gpu
def test_bounds_out_of_range():
    gen = torch.Generator().manual_seed(1)
    n = 300
    q, k, v = (x.to(DEV) for x in (randn(gen, n, 4, 64), randn(gen, n, 4, 64), randn(gen, n, 4, 64)))
    whole = K.prompt_attention(q, k, v, int32([0, n]))
    for begin in ([-5, 2 ** 31 - 1], [-2 ** 31, n + 1]):
        assert torch.equal(K.prompt_attention(q, k, v, int32(begin)), whole)
    out = torch.full_like(q, 7.0)
    K.prompt_attention(q, k, v, int32([200, 100, 50]), out=out)
    torch.cuda.synchronize()
    assert (out == 7).all()


@gpu
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (96, 24, 64), (96, 8, 128)])
@pytest.mark.parametrize("empty", [0, 30])
def test_prompts_on_another_stream_and_in_a_graph(hq, hkv, d, empty):
    gen = torch.Generator().manual_seed(6)
    n = 500
    q, k, v = (x.to(DEV) for x in (randn(gen, n, hq, d), randn(gen, n, hkv, d), randn(gen, n, hkv, d)))
    begin, out = int32([0] * empty + [0, 100, 500]), torch.zeros_like(q)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    other = K.prompt_attention(q, k, v, begin, stream=side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        K.prompt_attention(q, k, v, begin, out=out)
    for bounds in ([0, 100, 500], [0, 400, 500], [0, 0, 490], [0, 250, 250]):
        begin.copy_(int32([bounds[0]] * empty + bounds))
        out.fill_(7.0)
        graph.replay()
        eager = K.prompt_attention(q, k, v, begin, out=torch.full_like(q, 7.0))
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        if bounds == [0, 100, 500]:
            assert torch.equal(out, other)


def _prompts(**over):
    of = dict(q=P16, k=P16, v=P16, out=P16, seq_begin=P4, q_token=512, q_head=128, k_token=256, k_head=128, v_token=256, v_head=128, out_token=512,
              out_head=128, n_tokens=5, n_seqs=2, n_q_heads=4, n_kv_heads=2, head_dim=128, softmax_scale=0.0)
    of.update(over)
    return K.kvp_prompt_attention(K.KvpPrompts(**of))


def test_refusals():
    for bad in [dict(q=None), dict(k=P16 + 2), dict(v=None), dict(out=P16 + 8), dict(seq_begin=None), dict(seq_begin=P4 + 2), dict(q_token=516), dict(k_token=120),
                dict(v_token=-256), dict(out_token=1 << 23), dict(q_head=1 << 40), dict(k_head=12), dict(n_tokens=-1), dict(n_seqs=0), dict(n_seqs=4097),
                dict(n_q_heads=3), dict(n_q_heads=0), dict(n_kv_heads=0), dict(head_dim=96), dict(softmax_scale=-1.0), dict(softmax_scale=math.nan),
                dict(softmax_scale=math.inf), dict(out_token=256), dict(out_head=64), dict(n_tokens=2 ** 31 - 1, n_q_heads=256)]:
        assert _prompts(**bad) == K.KVP_EINVAL, bad
    assert K.lib().kvp_prompt_attention(None, None) == K.KVP_EINVAL
    assert _prompts(n_tokens=0, q=None, k=None, v=None, out=None) == K.KVP_OK


@gpu
def test_refusals_of_tensors():
    row = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16, device=DEV)
    good = dict(q=row(3, 4, 128), k=row(3, 2, 128), v=row(3, 2, 128), seq_begin=int32([0, 1, 3]))
    K.prompt_attention(**good)
    for bad in [dict(q=row(3, 3, 128)), dict(q=row(4, 4, 128)), dict(k=row(3, 2, 64)), dict(v=row(3, 4, 128)), dict(v=row(3, 2, 128).half()), dict(k=row(3, 2, 128).cpu()),
                dict(q=row(3, 128, 4).transpose(1, 2)), dict(seq_begin=int32([0, 3]).long()), dict(out=row(3, 4, 64)), dict(out=row(3, 1, 128).expand(3, 4, 128)),
                dict(q=row(3, 4, 32), k=row(3, 2, 32), v=row(3, 2, 32)), dict(q=row(3, 4, 132)[..., 4:])]:
        with pytest.raises(K.KvpError):
            K.prompt_attention(**dict(good, **bad))
    torch.cuda.synchronize()


@gpu
@pytest.mark.parametrize("e4m3", [False, True])
def test_prompts_pages_and_steps_together(e4m3):
    """A server's round of one layer: short prompts whole, a long one compressed as it is prefilled; all of them into pages; a few tokens of
    all together; and the compressed cache back into a kvp_cache that goes on."""
    gen = torch.Generator().manual_seed(13)
    hq, hkv, d, page, budget = 8, 2, 128, 32, 128
    lengths = [40, 1, 97]
    begin = [0, 40, 41, 138]
    q, k, v = (randn(gen, 138, h, d).to(DEV) for h in (hq, hkv, hkv))
    out = K.prompt_attention(q, k, v, int32(begin))
    ref, size, most = causal(q, k, v, begin, d ** -0.5)
    torch.cuda.synchronize()
    same(out, ref, size, most, d)
    cache = K.Cache(1, hq, hkv, d, budget, 64, [Segment(0, 1000, 0)], device=DEV)
    for t in range(0, 192, 64):
        cache.prefill_chunk(0, t, *(randn(gen, 64, h, d).to(DEV) for h in (hq, hkv, hkv)))
        cache.compact(0)
    ck, cv, token, weight, count, seen = cache.decode_ready(0)
    assert count == budget
    width = 8
    pages = K.Pages.empty(4 * width, hkv, d, page, e4m3, DEV)
    table = torch.randperm(4 * width, generator=gen).view(4, width).int().to(DEV)
    pages.write(k, v, int32(begin), table[:3].contiguous())
    pages.write(ck[:, :count].transpose(0, 1), cv[:, :count].transpose(0, 1), int32([0, count]), table[3:].contiguous())
    at = int32(lengths + [count])
    for step in range(3):
        q1, k1, v1 = (randn(gen, 4, h, d).to(DEV) for h in (hq, hkv, hkv))
        pages.write(k1, v1, int32([0, 1, 2, 3, 4]), table, first=at)
        at += 1
        out = pages.decode(q1, table, at)
        torch.cuda.synchronize()
        ref, size, most = reference(q1.double().cpu().numpy(), Pool(pages), table.cpu().numpy(), at.tolist(), pages.n_pages, page, d ** -0.5)
        check(out, ref, size, most, d)
        if not e4m3 and step == 0:                          # the one sequence that kvp_decode_step knows, too
            alone = cache.decode_step(0, q1[3], k1[3:], v1[3:])
            torch.cuda.synchronize()
            check(alone[None], ref[3:], size[3:], most, d)
    # back: e4m3 numbers are bf16 numbers, so a second time around nothing changes
    other = K.Cache(1, hq, hkv, d, budget, 64, [Segment(0, 1000, 0)], device=DEV)
    ok, ov, otoken, oweight, _, _ = other.decode_ready(0)
    pages.read(ok[:, :count].transpose(0, 1), ov[:, :count].transpose(0, 1), int32([0, count]), table[3:].contiguous())
    otoken.copy_(token), oweight.copy_(weight)
    other.set_state(0, count, seen)
    torch.cuda.synchronize()
    if not e4m3:
        assert torch.equal(ok, ck) and torch.equal(ov, cv)
    else:
        assert ((ok - ck).abs() <= ck.abs() * 2.0 ** -4 + ck.abs().amax(-1, keepdim=True) * 2.0 ** -17).all()       # half of 2^-9 for rows that fill more than 224
        held = Pool(pages)
        pages.write(ok[:, :count].transpose(0, 1), ov[:, :count].transpose(0, 1), int32([0, count]), table[3:].contiguous())
        torch.cuda.synchronize()
        pages.read(ok[:, :count].transpose(0, 1), ov[:, :count].transpose(0, 1), int32([0, count]), table[3:].contiguous())
        for n in range(count):
            for h in range(hkv):
                assert np.array_equal(held.row("k", int(table[3, n // page]), h, n % page), ok[h, n].double().cpu().numpy())
    other.prefill_chunk(0, seen, *(randn(gen, 64, h, d).to(DEV) for h in (hq, hkv, hkv)))
    other.compact(0)
    assert other.decode_ready(0)[4] == budget
    torch.cuda.synchronize()
    cache.close(), other.close()


@gpu
@pytest.mark.parametrize("n,hq,hkv", [(450, 4, 2), (450, 96, 48), (900, 24, 12)])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_far_before_a_number_that_is_not_finite_have_the_same_bits(d, n, hq, hkv):
    """Rows of the 64 that such a key is among may be taken again, with weights that are not rounded; those before them are not, nor other prompts, nor
    heads that read another KV head."""
    gen = torch.Generator().manual_seed(d + n)
    q, k, v = (x.to(DEV) for x in (randn(gen, n, hq, d), randn(gen, n, hkv, d), randn(gen, n, hkv, d)))
    begin = int32([0, 100, n])
    good = K.prompt_attention(q, k, v, begin)
    for row, upto in ((70, 64), (100 + 130, 100 + 128), (n - 1, n - 1 - (n - 101) % 64)):
        k2, v2 = k.clone(), v.clone()
        k2[row, 0, 3], v2[row, 0, 5] = math.nan, math.inf
        out = K.prompt_attention(q, k2, v2, begin)
        torch.cuda.synchronize()
        same_bits = torch.ones(n, hq, dtype=torch.bool, device=DEV)
        same_bits[upto:100 if row < 100 else n, :hq // hkv] = False
        assert torch.equal(out[same_bits], good[same_bits]) and not torch.isfinite(out[row, :hq // hkv]).all()


@gpu
@pytest.mark.parametrize("lengths", [(0, 3), (20, 70)])
def test_as_many_prompts_as_a_call_takes(lengths):
    gen = torch.Generator().manual_seed(lengths[1])
    lengths = [int(x) for x in torch.randint(*lengths, (K.KVP_MAX_SEQUENCES,), generator=gen)]
    lengths[1000:1300] = [0] * 300
    begin = np.concatenate([[0], np.cumsum(lengths)]).tolist()
    n = begin[-1]
    q, k, v = randn(gen, n, 2, 64), randn(gen, n, 1, 64), randn(gen, n, 1, 64)
    out = K.prompt_attention(q.to(DEV), k.to(DEV), v.to(DEV), int32(begin))
    torch.cuda.synchronize()
    ref, size, most = causal(q, k, v, begin, 0.125)
    assert np.isfinite(ref).all()
    same(out, ref, size, most, 64)
