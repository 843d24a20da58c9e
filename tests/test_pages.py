"""Pages: rows of K and V written into the pages of their sequences and read back, against the definition in 64 bits; refusals."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2604_16734_amd as K
from tests import gpu_util as U

DEV = "cuda:0"
gpu = pytest.mark.gpu


# ---- the definition
def to_e4m3(x):
    """(numbers, exponents + 127) of rows x [..., d] in 64 bits."""
    finite = np.isfinite(x)
    most = np.where(finite, np.abs(x), 0.0).max(axis=-1)
    exp = np.full(most.shape, -126)
    while True:
        more = most > 448.0 * np.exp2(exp)
        if not more.any():
            break
        exp = exp + more
    y = np.where(finite, x, 0.0) * np.exp2(-exp.astype(np.float64))[..., None]
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6))) - 3)       # four significant bits, multiples of 2^-9 below 2^-6
    return np.where(finite, np.round(y / step) * step, np.nan), (exp + 127).astype(np.int64)      # np.round: ties to even


class Pool:
    """What the pages hold, as numbers: [n_pages, heads, page, d] in 64 bits."""

    def __init__(self, pages):
        self.e4m3 = pages.k_exp is not None
        self.k, self.v = (t.double().cpu().numpy() for t in (pages.k, pages.v))
        if self.e4m3:
            self.k_exp, self.v_exp = (t.cpu().numpy().astype(np.int64) for t in (pages.k_exp, pages.v_exp))

    def row(self, name, page, head, offset):
        x = getattr(self, name)[page, head, offset]
        return x * np.exp2(float(getattr(self, name + "_exp")[page, head, offset]) - 127) if self.e4m3 else x

    def put(self, name, page, offset, rows):
        if self.e4m3:
            rows, exp = to_e4m3(rows)
            getattr(self, name + "_exp")[page, :, offset] = exp
        getattr(self, name)[page, :, offset] = rows

    def same(self, pages):
        other = Pool(pages)
        names = ("k", "v", "k_exp", "v_exp") if self.e4m3 else ("k", "v")
        return all(np.array_equal(getattr(self, n), getattr(other, n), equal_nan=n in "kv") for n in names)


def placed(begin, first, table, n_pages, page, n_tokens):
    """(token, page or None, offset) of every token that has a sequence."""
    for s in range(len(begin) - 1):
        for t in range(begin[s], min(begin[s + 1], n_tokens)):
            p = t - begin[s] + first[s]
            number = int(table[s, p // page]) if 0 <= p < table.shape[1] * page else -1
            yield t, number if 0 <= number < n_pages else None, p % page


def numbers(gen, *shape):
    return (torch.randn(shape, generator=gen) * torch.exp(3 * torch.randn(shape[:-1] + (1,), generator=gen))).to(torch.bfloat16)


def laid_out(x, how):
    """The rows x [n, heads, d] on the GPU with other strides."""
    x = x.to(DEV)
    if how == "heads":                                   # as a compressed cache holds them, with slots behind the last
        room = torch.full((x.shape[1], x.shape[0] + 5, x.shape[2]), 7.0, dtype=x.dtype, device=DEV)
        view = room[:, :x.shape[0]].transpose(0, 1)
    elif how == "projection":
        room = torch.full((x.shape[0], 3 * x.shape[1] + 1, x.shape[2]), 7.0, dtype=x.dtype, device=DEV)
        view = room[:, 1:2 * x.shape[1]:2] if x.shape[1] > 1 else room[:, 1:2]
    else:
        return x.contiguous(), None
    view.copy_(x)
    return view, room


def a_pool(gen, n_pages, heads, d, page, e4m3):
    """Pages full of numbers that no row has."""
    pages = K.Pages.empty(n_pages, heads, d, page, e4m3, DEV)
    for t in (pages.k, pages.v):
        t.copy_(torch.randint(1, 9, t.shape, generator=gen).to(torch.bfloat16))
    if e4m3:
        for t in (pages.k_exp, pages.v_exp):
            t.copy_(torch.randint(120, 130, t.shape, generator=gen))
    return pages


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


CASES = [
    # lengths, first, rows before and behind the sequences
    ([5], None, 0, 0),
    ([1], [0], 0, 0),
    ([33, 0, 1, 70], [0, 4, 15, 100], 0, 3),
    ([17, 16, 15], [1, 31, 16], 2, 9),
    ([0, 0], None, 0, 6),
    ([1 + i % 3 for i in range(70)] + [0] * 66 + [2], [(7 * i) % 90 for i in range(137)], 1, 1),      # more than two votes' worth
]


@gpu
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("d,heads,page,how", [(128, 8, 64, "rows"), (128, 3, 16, "heads"), (64, 1, 32, "projection"), (64, 5, 256, "rows"),
                                              (128, 1, 128, "projection"), (64, 2, 16, "heads")])
@pytest.mark.parametrize("lengths,first,before,behind", CASES)
def test_rows_go_into_pages_and_come_back(e4m3, d, heads, page, how, lengths, first, before, behind):
    gen = torch.Generator().manual_seed(len(lengths) + d + heads)
    begin = np.concatenate([[0], np.cumsum(lengths)]).astype(int) + before
    n = int(begin[-1]) + behind
    starts = first or [0] * len(lengths)
    width = max(-(-(f + m) // page) for f, m in zip(starts, lengths)) or 1
    n_pages = len(lengths) * width + 2
    table = torch.randperm(n_pages, generator=gen)[:len(lengths) * width].view(len(lengths), width).int()
    if len(lengths) > 1:                                  # pages that are not there, and a place outside of the table
        table[0, 0], table[-1, -1] = -1, n_pages
        width = max(1, width - 1) if len(lengths) == 3 else width
        table = table[:, :width].contiguous()
    pages = a_pool(gen, n_pages, heads, d, page, e4m3)
    expected = Pool(pages)
    k, v = numbers(gen, n, heads, d), numbers(gen, n, heads, d)
    (kd, _), (vd, _) = laid_out(k, how), laid_out(v, how)
    args = (int32(begin.tolist()), table.to(DEV), None if first is None else int32(first))
    pages.write(kd, vd, *args)
    for t, number, offset in placed(begin, starts, table, n_pages, page, n):
        if number is not None:
            expected.put("k", number, offset, k[t].double().numpy())
            expected.put("v", number, offset, v[t].double().numpy())
    assert expected.same(pages)
    # and back, into rows of another layout that hold something else
    other = {"rows": "heads", "heads": "projection", "projection": "rows"}[how]
    (kr, kroom), (vr, _) = laid_out(torch.full_like(k, 3.0), other), laid_out(torch.full_like(v, 3.0), other)
    pages.read(kr, vr, *args)
    k_ref, v_ref = np.full(k.shape, 3.0), np.full(v.shape, 3.0)
    for t, number, offset in placed(begin, starts, table, n_pages, page, n):
        for h in range(heads):
            k_ref[t, h] = 0.0 if number is None else expected.row("k", number, h, offset)
            v_ref[t, h] = 0.0 if number is None else expected.row("v", number, h, offset)
    assert np.array_equal(kr.double().cpu().numpy(), k_ref) and np.array_equal(vr.double().cpu().numpy(), v_ref)
    if kroom is not None:
        assert int((kroom == 7.0).sum()) == kroom.numel() - k.numel() + int((k_ref == 7.0).sum())          # what lies between the rows is left


@gpu
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("d,heads,n", [(128, 8, 5003), (64, 3, 22003), (128, 1, 33001)])
def test_many_rows(d, heads, n, e4m3):
    """More than the chip's waves take at once: several rows a wave, against the small calls that the other tests look at."""
    gen = torch.Generator().manual_seed(n)
    page, width = 64, -(-n // 64)
    k, v = (numbers(gen, n, heads, d).to(DEV) for _ in range(2))
    bounds = [0, 1, 1, n // 3, n - 700, n - 2]                                # the last two have no sequence
    table = torch.randperm(5 * width, generator=gen).view(5, width).int().to(DEV)
    first, many, few = int32([3, 0, 5, 0, 100]), *(a_pool(torch.Generator().manual_seed(1), 5 * width, heads, d, page, e4m3) for _ in range(2))
    many.write(k, v, int32(bounds), table, first)
    for s in range(5):
        for t in range(bounds[s], bounds[s + 1], 2000):
            m = min(2000, bounds[s + 1] - t)
            few.write(k[t:t + m], v[t:t + m], int32([0, m]), table[s:s + 1], int32([int(first[s]) + t - bounds[s]]))
    torch.cuda.synchronize()
    for name in ("k", "v", "k_exp", "v_exp")[:4 if e4m3 else 2]:
        assert torch.equal(getattr(many, name).view(torch.uint8), getattr(few, name).view(torch.uint8))
    kr, vr = torch.full_like(k, 3.0), torch.full_like(v, 3.0)
    many.read(kr, vr, int32(bounds), table, first)
    torch.cuda.synchronize()
    assert (kr[n - 2:] == 3).all() and (vr[n - 2:] == 3).all()
    for s in range(5):
        for t in range(bounds[s], bounds[s + 1], 2000):
            m = min(2000, bounds[s + 1] - t)
            ks, vs = torch.empty_like(k[:m]), torch.empty_like(v[:m])
            few.read(ks, vs, int32([0, m]), table[s:s + 1], int32([int(first[s]) + t - bounds[s]]))
            assert torch.equal(ks, kr[t:t + m]) and torch.equal(vs, vr[t:t + m])


@gpu
def test_e4m3_of_every_kind_of_row():
    """Every bf16 number, in rows whose largest magnitude is at most 2^r times theirs; zeros, infinities, NaNs; ties."""
    d, page = 64, 64
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    rows = [bits.view(-1, d)]                                                 # neighbours in size: one exponent, all 64 magnitudes
    rows += [bits.view(-1, d).flip(0).reshape(d, -1).T.contiguous().view(-1, d)]      # all exponents beside each other
    small = bits[(bits.abs() < 2.0 ** -100) & torch.isfinite(bits)]
    rows += [small[:small.numel() // d * d].view(-1, d)]
    x = torch.cat(rows)
    n = x.shape[0]
    x = torch.cat([x, torch.zeros(64 - n % 64, d, dtype=torch.bfloat16)]).view(-1, 1, d)
    pages = K.Pages.empty(x.shape[0] // page, 1, d, page, True, DEV)
    table = torch.arange(x.shape[0] // page, dtype=torch.int32, device=DEV).view(1, -1)
    begin = int32([0, x.shape[0]])
    pages.write(x.to(DEV), x.flip(0).to(DEV), begin, table)
    y, exp = to_e4m3(x[:, 0].double().numpy())
    held = Pool(pages)
    assert np.array_equal(held.k.reshape(-1, d), y, equal_nan=True) and np.array_equal(held.k_exp.reshape(-1), exp)
    assert np.array_equal(held.v.reshape(-1, d), y[::-1], equal_nan=True)
    back = torch.empty_like(x, device=DEV)
    pages.read(back, torch.empty_like(back), begin, table)
    ref = y * np.exp2(exp.astype(np.float64) - 127)[:, None]
    top = np.abs(ref) == 2.0 ** 128           # what 1.9375 2^127 and more round to with four bits: no bf16 number, an infinity
    assert top.any() and (np.abs(ref[~top & np.isfinite(ref)]) < 2.0 ** 128).all()
    ref[top] *= np.inf
    got = back[:, 0].double().cpu().numpy()
    assert np.array_equal(got, ref, equal_nan=True)
    # what the format promises: half a step of four significant bits, or of the smallest step
    finite = np.isfinite(x[:, 0].double().numpy()) & ~top
    err, size = np.abs(got - x[:, 0].double().numpy()), np.abs(x[:, 0].double().numpy())
    assert (err[finite] <= np.maximum(size * 2.0 ** -4, np.broadcast_to(np.exp2(exp - 127.0 - 10)[:, None], size.shape))[finite]).all()


@gpu
def test_beyond_32_bits_of_a_pool():
    page, heads, d = 256, 8, 128
    n_pages = (1 << 32) // (page * heads * d * 2) + 3                         # K alone passes 4 GiB
    pages = K.Pages.empty(n_pages, heads, d, page, False, DEV)
    gen = torch.Generator().manual_seed(4)
    k, v = (numbers(gen, 300, heads, d).to(DEV) for _ in range(2))
    table, begin = int32([[n_pages - 1, n_pages - 2]]), int32([0, 300])
    pages.k[:2].zero_()
    pages.write(k, v, begin, table)
    assert torch.equal(pages.k[n_pages - 1].transpose(0, 1), k[:256]) and torch.equal(pages.v[n_pages - 2].transpose(0, 1)[:44], v[256:])
    assert not pages.k[:2].any()
    kr, vr = torch.zeros_like(k), torch.zeros_like(v)
    pages.read(kr, vr, begin, table)
    assert torch.equal(kr, k) and torch.equal(vr, v)


@gpu
def test_pages_on_another_stream_and_in_a_graph():
    gen = torch.Generator().manual_seed(5)
    pages = a_pool(gen, 9, 2, 128, 64, True)
    k, v = (numbers(gen, 100, 2, 128).to(DEV) for _ in range(2))
    begin, table, first = int32([0, 60, 100]), int32([[3, 5, 1], [7, 2, 0]]), int32([10, 90])
    back = [torch.zeros_like(k) for _ in range(2)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    pages.write(k, v, begin, table, first, stream=side)
    with torch.cuda.stream(side):
        pages.read(*back, begin, table, first)
    torch.cuda.synchronize()
    expected = [b.clone() for b in back]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pages.write(k, v, begin, table, first)
        pages.read(*back, begin, table, first)
    for shift in (0, 3, 21):
        first.copy_(int32([10 + shift, 90 - shift]))                          # the graph reads it anew
        for b in back:
            b.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(b, e) for b, e in zip(back, expected))
        other = [torch.zeros_like(k) for _ in range(2)]
        pages.read(*other, begin, table, first)
        assert all(torch.equal(b, e) for b, e in zip(other, expected))


# ---- refusals: before anything is enqueued, so they need no GPU
P16, P4 = 0x10000, 0x20004


def _pages(**over):
    of = dict(k=P16, v=P16, k_exp=None, v_exp=None, format=K.KVP_PAGE_BF16, n_pages=10, n_kv_heads=2, page_size=64, head_dim=128)
    if over.get("format") == K.KVP_PAGE_E4M3:
        of.update(k_exp=P4, v_exp=P4)
    of.update(over)
    return K.KvpPages(**of)


def _some_rows(**over):
    of = dict(k=P16, v=P16, k_token=256, k_head=128, v_token=256, v_head=128, n_tokens=3)
    of.update(over)
    return K.KvpRows(**of)


def _call(call, pages=None, rows=None, begin=P4, table=P4, width=4, first=None, n_seqs=2):
    return call(pages or _pages(), rows or _some_rows(), begin, table, width, first, n_seqs)


BAD_PAGES = [dict(k=None), dict(v=None), dict(k=P16 + 8), dict(format=2), dict(format=-1), dict(n_pages=0), dict(n_kv_heads=0),
             dict(page_size=8), dict(page_size=48), dict(page_size=512), dict(page_size=0), dict(head_dim=96), dict(k_exp=P4, v_exp=P4),
             dict(format=K.KVP_PAGE_E4M3, k_exp=None), dict(format=K.KVP_PAGE_E4M3, v_exp=P4 + 1),
             dict(n_pages=2 ** 31 - 1, n_kv_heads=2 ** 20)]


@pytest.mark.parametrize("call", [K.kvp_page_write, K.kvp_page_read])
def test_refusals(call):
    for bad in BAD_PAGES:
        assert _call(call, _pages(**bad)) == K.KVP_EINVAL, bad
    for bad in [dict(k=None), dict(v=P16 + 2), dict(k_token=-8), dict(v_head=4), dict(k_token=1 << 23), dict(k_head=1 << 40), dict(n_tokens=-1),
                dict(n_tokens=1 << 30)]:
        assert _call(call, rows=_some_rows(**bad)) == K.KVP_EINVAL, bad
    for bad in [dict(begin=None), dict(begin=P4 + 1), dict(table=None), dict(width=0), dict(width=(1 << 24) + 1), dict(first=P4 + 2), dict(n_seqs=0),
                dict(n_seqs=K.KVP_MAX_SEQUENCES + 1)]:
        assert _call(call, **bad) == K.KVP_EINVAL, bad
    L = K.lib()
    entry = getattr(L, call.__name__)
    assert entry(None, ctypes.byref(_some_rows()), P4, P4, 4, None, 2, None) == K.KVP_EINVAL
    assert entry(ctypes.byref(_pages()), None, P4, P4, 4, None, 2, None) == K.KVP_EINVAL
    assert _call(call, rows=_some_rows(n_tokens=0, k=None, v=None)) == K.KVP_OK


def test_rows_that_are_written_do_not_overlap():
    for bad in [dict(k_token=128), dict(v_head=64), dict(k_token=0), dict(k_token=128, k_head=256)]:
        assert _call(K.kvp_page_read, rows=_some_rows(**bad)) == K.KVP_EINVAL, bad


def test_refusals_in_python():
    with pytest.raises(K.KvpError):
        K.Pages(torch.zeros(2, 2, 64, 128, dtype=torch.bfloat16), torch.zeros(2, 2, 64, 128, dtype=torch.bfloat16))       # not on a GPU
    with pytest.raises(K.KvpError):
        K.Pages(torch.zeros(2, 2, 64, 128), torch.zeros(2, 2, 64, 128))


@gpu
def test_refusals_of_tensors():
    pages = K.Pages.empty(4, 2, 128, 64, False, DEV)
    row = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16, device=DEV)
    good = dict(k=row(3, 2, 128), v=row(3, 2, 128), seq_begin=int32([0, 1, 3]), table=int32([[0], [1]]), first=int32([0, 0]))
    pages.write(**good)
    for bad in [dict(k=row(3, 2, 64)), dict(v=row(4, 2, 128)), dict(k=row(3, 2, 128).float()), dict(k=row(3, 2, 128).cpu()), dict(k=row(3, 128, 2).transpose(1, 2)),
                dict(k=row(3, 2, 132)[..., 2:130]), dict(seq_begin=int32([0, 1, 3]).long()), dict(seq_begin=int32([0, 0, 1, 1, 3, 3])[::2]),
                dict(table=int32([[0, 1], [1, 2]])[:, :1]), dict(table=int32([[0]])), dict(table=int32([0, 1])), dict(first=int32([0]))]:
        with pytest.raises(K.KvpError):
            pages.write(**dict(good, **bad))
    with pytest.raises(K.KvpError):
        pages.read(**dict(good, k=row(1, 2, 128).expand(3, 2, 128)))
    with pytest.raises(K.KvpError):
        K.Pages(row(4, 2, 64, 128), row(4, 2, 64, 128), torch.zeros(4, 2, 64, dtype=torch.uint8, device=DEV))
    with pytest.raises(K.KvpError):
        K.Pages(row(4, 2, 64, 128), row(4, 2, 64, 128).transpose(0, 1).contiguous().transpose(0, 1))


def test_tensors_of_pages_cannot_be_exchanged():
    for name in ("k", "v", "k_exp", "v_exp", "device", "n_pages", "n_kv_heads", "page_size", "head_dim", "of"):
        found = getattr(K.Pages, name)
        assert isinstance(found, property) and found.fset is None, name


@gpu
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("native", [True, False])
def test_pages_whose_memory_is_another_one(e4m3, native):
    """The calls have the tensors' addresses: after resize_ or set_ these would be those of memory that is not theirs any more."""
    row = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16, device=DEV)
    stream = None if native else torch.cuda.current_stream()
    args = dict(seq_begin=int32([0, 1, 3]), table=int32([[0], [1]]), stream=stream)
    for name in ("k", "v", "k_exp", "v_exp")[:4 if e4m3 else 2]:
        for change in (lambda t: t.resize_(2 * t.numel()), lambda t: t.set_(torch.zeros_like(t))):
            pages = K.Pages.empty(4, 2, 128, 64, e4m3, DEV)
            k, v, q, out = row(3, 2, 128), row(3, 2, 128), row(2, 4, 128), row(2, 4, 128)
            calls = [lambda: pages.write(k, v, **args), lambda: pages.read(k, v, **args),
                     lambda: pages.decode(q, args["table"], int32([1, 2]), out=out, stream=stream), lambda: pages.decode(q, args["table"], int32([1, 2]), stream=stream)]
            for call in calls:
                call()
            with pytest.raises(AttributeError):
                setattr(pages, name, torch.zeros_like(getattr(pages, name)))
            pages.of.head_dim = 64                                              # of a copy
            for call in calls:
                call()
            torch.cuda.synchronize()
            change(getattr(pages, name))
            for call in calls:
                with pytest.raises(K.KvpError):
                    call()
    torch.cuda.synchronize()


@gpu
@pytest.mark.parametrize("e4m3", [False, True])
def test_as_many_sequences_as_a_call_takes(e4m3):
    gen = torch.Generator().manual_seed(21)
    n_seqs, heads, d, page, width = K.KVP_MAX_SEQUENCES, 3, 64, 16, 2
    lengths = [int(x) for x in torch.randint(0, 4, (n_seqs,), generator=gen)]
    lengths[200:600] = [0] * 400
    begin = np.concatenate([[0], np.cumsum(lengths)]).astype(int) + 5
    first = [int(x) for x in torch.randint(0, 28, (n_seqs,), generator=gen)]
    n, n_pages = int(begin[-1]) + 2, n_seqs * width
    table = torch.randperm(n_pages, generator=gen).view(n_seqs, width).int()
    pages = a_pool(gen, n_pages, heads, d, page, e4m3)
    expected = Pool(pages)
    k, v = numbers(gen, n, heads, d), numbers(gen, n, heads, d)
    args = (int32(begin.tolist()), table.to(DEV), int32(first))
    pages.write(k.to(DEV), v.to(DEV), *args)
    k_ref, v_ref = np.full(k.shape, 3.0), np.full(v.shape, 3.0)
    for t, number, offset in placed(begin, first, table, n_pages, page, n):
        expected.put("k", number, offset, k[t].double().numpy())
        expected.put("v", number, offset, v[t].double().numpy())
        for h in range(heads):
            k_ref[t, h], v_ref[t, h] = expected.row("k", number, h, offset), expected.row("v", number, h, offset)
    assert expected.same(pages)
    kr, vr = torch.full_like(k, 3.0).to(DEV), torch.full_like(v, 3.0).to(DEV)
    pages.read(kr, vr, *args)
    assert np.array_equal(kr.double().cpu().numpy(), k_ref) and np.array_equal(vr.double().cpu().numpy(), v_ref)
