"""The native way of the calls of many sequences: what it hands on, and what it leaves to Python, for tensors on the CPU and an entry point that
only looks at its arguments."""
import ctypes
import importlib.util
import os
import subprocess
import sys

import pytest
import torch

import paper_2604_16734_amd as K
from paper_2604_16734_amd import build as build_module

BF16 = torch.bfloat16
P, I, L, F, Z = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
ROWS = ctypes.CFUNCTYPE(ctypes.c_int, P, ctypes.POINTER(K.KvpRows), P, P, I, P, I, P)
DECODE = ctypes.CFUNCTYPE(ctypes.c_int, P, P, L, L, I, P, I, P, I, F, P, P, Z, P)
PROMPT = ctypes.CFUNCTYPE(ctypes.c_int, ctypes.POINTER(K.KvpPrompts), P)


@pytest.fixture(scope="module")
def module(tmp_path_factory):
    path = build_module.build_fast_calls(os.path.join(str(tmp_path_factory.mktemp("fast_calls")), "_fast_calls.so"),
                                         ["KVP_TENSOR_DEVICE=c10::DeviceType::CPU"])
    spec = importlib.util.spec_from_file_location("_fast_calls", path)
    found = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(found)
    return found


def address(entry):
    return ctypes.cast(entry, P).value


def fields(struct):
    return {name: getattr(struct, name) for name, _ in struct._fields_}


def int32(*x):
    return torch.tensor(x, dtype=torch.int32)


def left(call, good, others, taken):
    """One argument at a time of a call that is taken."""
    n = len(taken)
    for at, values in others:
        for other in values:
            assert call(*(good[:at] + [other] + good[at + 1:])) is None, (at, other)
    assert len(taken) == n
    for wrong in (good[:-1], good + [None]):
        with pytest.raises(TypeError):
            call(*wrong)


INTS = [None, 1.0, "1", 1 << 40]
ADDRESSES = [None, "1", -1, 1 << 64]


def rows_of(*shape):
    return torch.zeros(*shape, dtype=BF16)


def odd(x):
    """Tensors unlike x [tokens, heads, d] in one respect."""
    wide = torch.zeros(*x.shape[:2], 2 * x.shape[2], dtype=x.dtype)
    return [None, x.float(), x[1:], x[:, 1:], x[..., :-64], x[None], x[0], wide[..., ::2], x.transpose(1, 2), x.to_sparse(), x.to("meta"), x.numpy]


def test_rows(module):
    taken = []
    entry = ROWS(lambda pages, rows, begin, table, width, first, n_seqs, stream: taken.append((pages, fields(rows[0]), begin, table, width, first, n_seqs, stream)) or 7)
    k, v = rows_of(3, 5, 128)[:, 1:3], rows_of(2, 9, 128)[:, :3].transpose(0, 1)
    begin, table, first = int32(0, 1, 3), torch.zeros(2, 6, dtype=torch.int32), int32(4, 5)
    good = [address(entry), 11, 2, 128, -1, 13, k, v, begin, table, first]
    assert module.page_rows(*good) == 7
    assert taken == [(11, dict(k=k.data_ptr(), v=v.data_ptr(), k_token=640, k_head=128, v_token=128, v_head=1152, n_tokens=3), begin.data_ptr(), table.data_ptr(), 6,
                      first.data_ptr(), 2, 13)]
    assert module.page_rows(*good[:-1], None) == 7 and taken[-1][5] is None
    # distances of one token or head mean nothing; no tokens, no address
    one = rows_of(1, 2, 128).as_strided((1, 2, 128), (3, 128, 1))
    assert module.page_rows(*good[:6], one, one, begin, table, None) == 7 and taken[-1][1]["k_token"] == 0
    none = rows_of(0, 2, 128)
    assert module.page_rows(*good[:6], none, none, begin, table, None) == 7 and taken[-1][1]["n_tokens"] == 0 and taken[-1][1]["k"] is None
    left(module.page_rows, good, [(0, ADDRESSES + [0]), (1, ADDRESSES + [0]), (2, INTS + [3]), (3, INTS + [64]), (4, INTS + [0]), (5, ADDRESSES), (6, odd(k)), (7, odd(v)),
                                  (8, [None, begin[1:], begin.long(), int32(0, 0, 1, 1, 3, 3)[::2], begin[None]]),
                                  (9, [None, table[1:], table[0], table.long(), torch.zeros(2, 7, dtype=torch.int32)[:, :6]]),
                                  (10, [0, first[1:], first.long(), first[None], int32(1, 2, 3, 4)[::2]])], taken)


@pytest.mark.parametrize("own", [False, True])
def test_decode(module, own):
    taken = []
    entry = DECODE(lambda *args: taken.append(args) or 7)
    q, out, table, lengths = rows_of(2, 9, 128)[:, :8:2], rows_of(2, 4, 128), torch.zeros(2, 6, dtype=torch.int32), int32(1, 2)
    room = 4096 if own else torch.zeros(4096, dtype=torch.uint8)
    good = [address(entry), 11, 4, 128, -1, 13, q, table, lengths, out, room, 0.25]
    assert module.paged_decode(*good) == 7
    assert taken[0][:11] == (11, q.data_ptr(), 1152, 256, 4, table.data_ptr(), 6, lengths.data_ptr(), 2, 0.25, out.data_ptr())
    assert taken[0][12:] == (4096, 13) and (taken[0][11] == room.data_ptr() if not own else taken[0][11] % 16 == 0)
    left(module.paged_decode, good, [(0, ADDRESSES + [0]), (1, ADDRESSES + [0]), (2, INTS + [3]), (3, INTS + [64]), (4, INTS + [0]), (5, ADDRESSES), (6, odd(q)),
                                     (7, [None, table[1:], table[0], table.long(), torch.zeros(2, 7, dtype=torch.int32)[:, :6]]),
                                     (8, [None, lengths[1:], lengths.long(), lengths[None], int32(1, 2, 3, 4)[::2]]), (9, odd(out) + [rows_of(4, 2, 128).transpose(0, 1)]),
                                     (10, [None, 1.0, torch.zeros(64), torch.zeros(64, dtype=torch.uint8)[::2]]), (11, [None, 1, "1"])], taken)


def test_prompt(module):
    taken = []
    entry = PROMPT(lambda prompts, stream: taken.append((fields(prompts[0]), stream)) or 7)
    q, k, v, out = rows_of(3, 9, 64)[:, :8:2], rows_of(3, 2, 64), rows_of(2, 7, 64)[:, 2:5].transpose(0, 1), rows_of(4, 5, 64)[:, 1:4].transpose(0, 1)
    begin = int32(0, 1, 3)
    good = [address(entry), -1, 13, q, k, v, begin, out, 0.5]
    assert module.prompt(*good) == 7
    assert taken == [(dict(q=q.data_ptr(), k=k.data_ptr(), v=v.data_ptr(), out=out.data_ptr(), seq_begin=begin.data_ptr(), q_token=576, q_head=128, k_token=128, k_head=64,
                           v_token=64, v_head=448, out_token=64, out_head=320, n_tokens=3, n_seqs=2, n_q_heads=4, n_kv_heads=2, head_dim=64, softmax_scale=0.5), 13)]
    wide = [rows_of(3, 4, 128), rows_of(3, 2, 128)]
    left(module.prompt, good, [(0, ADDRESSES + [0]), (1, INTS + [0]), (2, ADDRESSES), (3, [q[1:], q[0], q.float(), wide[0], q.transpose(1, 2), None]),
                               (4, [k[1:], k[0], k.float(), wide[1], rows_of(3, 4, 64), None]), (5, [v[1:], v[:, 1:], v.float(), wide[1], None]),
                               (6, [None, begin.long(), begin[None], begin[:0], int32(0, 0, 1, 1, 3, 3)[::2]]),
                               (7, [out[1:], out[:, 1:], out.float(), wide[0], None]), (8, [None, 1, "1"])], taken)


NO_ROOM = """
import importlib.util, os, resource, sys
sys.path.insert(0, %r)
from tests import test_fast_calls_of_many as T
spec = importlib.util.spec_from_file_location("_fast_calls", %r)
module = importlib.util.module_from_spec(spec)
spec.loader.exec_module(module)
name, at, taken = %r, %d, []
entry = {"page_rows": T.ROWS, "paged_decode": T.DECODE, "prompt": T.PROMPT}[name](lambda *args: taken.append(args) or 7)
args = T.large(name, T.address(entry))
whole = args[at]
args[at] = T.torch._lazy_clone(whole)
with open("/proc/self/statm") as f:
    size = int(f.read().split()[0]) * resource.getpagesize()
resource.setrlimit(resource.RLIMIT_AS, (size + (1 << 28), resource.RLIM_INFINITY))
found = getattr(module, name)(*args)
print("left" if found is None and not taken else (found, taken), flush=True)
os._exit(0)          # (torch ends the process when it frees a clone that it could not copy)
"""


def large(name, entry):
    """Arguments whose bf16 tensors and workspace have 1 GiB each, none of which is touched."""
    new, begin, d = lambda *shape: torch.empty(*shape, dtype=BF16), int32(0, 1, 2), 1 << 27
    if name == "page_rows":
        return [entry, 11, 2, d, -1, 13, new(2, 2, d), new(2, 2, d), begin, torch.zeros(2, 6, dtype=torch.int32), int32(4, 5)]
    if name == "paged_decode":
        return [entry, 11, 2, d, -1, 13, new(2, 2, d), torch.zeros(2, 6, dtype=torch.int32), int32(1, 2), new(2, 2, d), torch.empty(1 << 30, dtype=torch.uint8), 0.25]
    return [entry, -1, 13, new(2, 2, d), new(2, 2, d), new(2, 2, d), begin, new(2, 2, d), 0.5]


@pytest.mark.parametrize("name,at", [("paged_decode", 9), ("paged_decode", 10), ("paged_decode", 6), ("page_rows", 6), ("page_rows", 7), ("prompt", 3), ("prompt", 7)])
def test_tensors_that_have_to_be_copied_and_no_room_for_it(module, name, at):
    """Torch copies a lazy clone when its address is asked for, and throws where it cannot: no exception may leave the module (a process of its
    own, which it would end)."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    run = subprocess.run([sys.executable, "-c", NO_ROOM % (root, module.__file__, name, at)], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.strip() == "left", (run.returncode, run.stderr[-500:])


@pytest.mark.parametrize("name", ["page_rows", "paged_decode"])
def test_memory_of_the_pages(module, name):
    """Pages by their tensors: taken while the tensors' memory is what the struct says, and left when one has been given other memory."""
    taken = []
    entry = {"page_rows": ROWS, "paged_decode": DECODE}[name](lambda *args: taken.append(args[0]) or 7)
    if name == "page_rows":
        rest = [2, 128, -1, 13, rows_of(3, 2, 128), rows_of(3, 2, 128), int32(0, 1, 3), torch.zeros(2, 6, dtype=torch.int32), None]
    else:
        rest = [4, 128, -1, 13, rows_of(2, 4, 128), torch.zeros(2, 6, dtype=torch.int32), int32(1, 2), rows_of(2, 4, 128), 4096, 0.25]
    call = lambda pages: getattr(module, name)(address(entry), pages, *rest)
    for n in (2, 4):
        new = lambda: [torch.zeros(4, 2, 16, 64, dtype=torch.uint8) for _ in range(2)] + [torch.zeros(4, 2, 16, dtype=torch.uint8) if n == 4 else None for _ in range(2)]
        tensors = new()
        of = K.KvpPages(*(t.data_ptr() if t is not None else None for t in tensors), 1 if n == 4 else 0, 4, 2, 16, 64)
        at = ctypes.addressof(of)
        assert call((at, *tensors)) == 7 and taken.pop() == at
        assert call(at) == 7 and taken.pop() == at
        for bad in [(at, *tensors[:3]), (at, *tensors, None), (at, *tensors[1::-1], *tensors[2:]), (0, *tensors), (None, *tensors), [at, *tensors], (at, 1, *tensors[1:]),
                    (at, *new()), (at, None, *tensors[1:]), (at, *tensors[:2], tensors[0], tensors[3])]:
            assert call(bad) is None and not taken
        for i in range(n):
            for other in (lambda t: t.resize_(1 << 20), lambda t: t.set_(torch.zeros_like(t)), lambda t: setattr(t, "data", torch.zeros_like(t)),
                          lambda t: t.untyped_storage().resize_(1 << 22)):
                tensors = new()
                of.k, of.v, of.k_exp, of.v_exp = (t.data_ptr() if t is not None else None for t in tensors)
                assert call((at, *tensors)) == 7 and taken.pop() == at
                other(tensors[i])
                assert call((at, *tensors)) is None and not taken, i
