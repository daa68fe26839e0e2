"""The paged cache's host side, without a GPU: configurations, sizes, NULL arguments, the binding's marshalling, and what the compiler
makes of the kernels that exchange partials."""
import ctypes
import re
import types

import pytest

import paper_2504_03661_amd as P
from paper_2504_03661_amd import binding as B
from tests.test_exchange_codegen_cpu import assembly, kernels


def good(**kw):
    c = P.PQPagedConfig(max_seqs=64, max_tokens=8192, n_q_heads=32, n_kv_heads=8, n_blocks=4096, max_blocks=512)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


@pytest.mark.parametrize("changes,status", [
    ({}, 0),
    ({"dtype": P.PQ_F32}, 0),
    ({"dtype": P.PQ_BF16}, 0),
    ({"head_dim": 64, "block_tokens": 64}, 0),
    ({"n_q_heads": 8 * 37}, 0),
    ({"max_seqs": 4096, "max_tokens": 1 << 20}, 0),
    ({"max_seqs": 0}, -2),
    ({"max_tokens": -1}, -2),
    ({"n_q_heads": 12}, -2),                                    # Hq % Hkv
    ({"n_kv_heads": 0}, -2),
    ({"n_blocks": 0}, -2),
    ({"max_blocks": 0}, -2),
    ({"dtype": 3}, -2),
    ({"device": -1}, -2),
    ({"reserved": 1}, -2),
    ({"head_dim": 96}, -3),
    ({"block_tokens": 48}, -3),
    ({"block_tokens": 128}, -3),
    ({"max_seqs": 4097}, -3),
    ({"max_tokens": (1 << 20) + 1}, -3),
    ({"n_q_heads": 1032}, -3),
    ({"n_q_heads": 1024, "max_tokens": 1 << 18}, 0),
    ({"n_q_heads": 1024, "max_tokens": (1 << 18) + 1}, -3),     # more threads than a launch has
    ({"n_blocks": 1 << 27}, -3),                                # slots beyond 31 bits
    ({"n_blocks": (1 << 27) - 1}, 0),
    ({"max_blocks": (1 << 20) + 1}, -3),                        # sequences longer than 2^24 tokens
    ({"max_blocks": 1 << 20}, 0),
])
def test_validate_config(changes, status):
    c = good(**changes)
    assert P.pq_paged_validate_config(c) == status
    if status:
        out = ctypes.c_void_p()
        assert P.load_library().pq_paged_create(ctypes.byref(c.c_struct()), ctypes.byref(out)) == status     # before any HIP call
        assert out.value is None
        with pytest.raises(P.PQAttnError):
            P.pq_paged_cache_bytes(c)
    else:
        assert P.pq_paged_cache_bytes(c) == c.n_blocks * c.n_kv_heads * c.block_tokens * c.head_dim


def test_the_other_contexts_do_not_take_bf16():
    assert P.pq_attn_validate_config(P.PQAttnConfig(batch=1, n_q_heads=1, n_kv_heads=1, max_context=64, dtype=P.PQ_BF16)) == -2


def test_null_arguments_are_rejected_without_a_gpu():
    lib = P.load_library()
    assert lib.pq_paged_validate_config(None) == -1
    assert lib.pq_paged_cache_bytes(None) == -1
    assert lib.pq_paged_create(None, None) == -1
    out = ctypes.c_void_p()
    assert lib.pq_paged_create(None, ctypes.byref(out)) == -1
    assert lib.pq_paged_destroy(None) == -1
    assert lib.pq_paged_device_error(None, None) == -1
    for name in ("plan", "append", "read", "decode", "prefill"):
        f = getattr(lib, "pq_paged_" + name)
        assert f(*[1 if t in (ctypes.c_int32, ctypes.c_int64) else 1.0 if t is ctypes.c_float else None for t in f.argtypes]) == -1


class Tensor:
    def __init__(self, at):
        self.at = at

    def data_ptr(self):
        return self.at


HIGH = 0xFFFF_8000_0000_1000      # an address with the top bit set
SAMPLES = {"n_seqs": (3, 2 ** 31 - 1, -1), "n_tokens": (7, 0, -2 ** 31), "n_rows": (5, 0, -1), "kv_stride": (256, 2 ** 40, -8),
           "q_stride": (512, 2 ** 31, -1), "scale": (0.125, -2.0, 0.0)}


def calls():
    import inspect
    for name in ("plan", "append", "read", "decode", "prefill"):
        f = getattr(B, "pq_paged_" + name)
        yield name, f, [p for p in inspect.signature(f).parameters if p not in ("ctx", "stream")]


@pytest.mark.parametrize("module", [True, False], ids=["extension module", "ctypes"])
def test_arguments_arrive_as_passed(monkeypatch, module):
    lib = B.load_library()
    if module and B._calls is None:
        pytest.skip("the extension module is not built here")
    for name, f, names in calls():
        seen = []
        kind = ctypes.CFUNCTYPE(ctypes.c_int32, *getattr(lib, "pq_paged_" + name).argtypes)
        fn = kind(lambda *a: seen.append(a) or 0)
        with monkeypatch.context() as m:
            if module:
                m.setitem(B._paged_at, name, ctypes.cast(fn, ctypes.c_void_p).value)
            else:
                m.setattr(B, "_calls", None)
                m.setattr(B, "_lib", types.SimpleNamespace(**{"pq_paged_" + name: fn}))
            for k in range(3):
                given = [SAMPLES[n][k] if n in SAMPLES else [Tensor(HIGH + 16 * i), 8 + i, None][(i + k) % 3] for i, n in enumerate(names)]
                f(HIGH, *given, stream=77)
                plain = [x.at if isinstance(x, Tensor) else x for x in given]
                assert seen.pop() == (HIGH, *plain, 77), name
            with pytest.raises((TypeError, AttributeError)):
                f(HIGH, *[object() for _ in names], stream=0)
            assert not seen
        failing = kind(lambda *a: -4)
        with monkeypatch.context() as m:
            if module:
                m.setitem(B._paged_at, name, ctypes.cast(failing, ctypes.c_void_p).value)
            else:
                m.setattr(B, "_calls", None)
                m.setattr(B, "_lib", types.SimpleNamespace(**{"pq_paged_" + name: failing, "pq_status_string": lib.pq_status_string}))
            with pytest.raises(P.PQAttnError) as e:
                f(0, *[SAMPLES[n][0] if n in SAMPLES else None for n in names], stream=0)
            assert e.value.status == -4


@pytest.fixture(scope="module")
def decode_kernels(tmp_path_factory):
    return assembly("pq_paged_decode.hip", tmp_path_factory.mktemp("asm"))


def test_partials_travel_with_sc1_and_the_ticket_is_a_device_atomic(decode_kernels):
    """The argument of the split exchange (pq_device_utils.h) for the paged decode: its agent-scope stores and loads pass the XCD's
    own cache, and the wait stands between the stores and the ticket."""
    ks = {k: v for k, v in kernels(decode_kernels).items() if "pq_paged_decode_kernel" in k}
    assert len(ks) == 6
    for name, body in ks.items():
        ticket = re.search(r"global_atomic_add\w* .*\bsc0\b", body)
        assert ticket, name
        stores = [m.start() for m in re.finditer(r"global_store_dwordx2 .*\bsc1\b", body)]
        loads = [m.start() for m in re.finditer(r"global_load_dwordx2 .*\bsc1\b", body)]
        assert stores and loads, name
        assert max(stores) < ticket.start(), name
        assert re.search(r"s_waitcnt vmcnt\(0\)", body[max(stores):ticket.start()]), name
        assert any(at > ticket.start() for at in loads), name


@pytest.mark.parametrize("source", ["pq_paged_decode.hip", "pq_paged_few.hip", "pq_paged_prefill.hip", "pq_paged_cache.hip"])
def test_no_kernel_spills_what_it_multiplies(source, tmp_path):
    """fp16 and bf16 kernels keep everything in registers; the fp32 ones, with operands in two parts, all but a few."""
    text = assembly(source, tmp_path)
    spills = {k: int(v) for k, v in re.findall(r"\.name:\s+(\S+)\s.*?\.vgpr_spill_count:\s+(\d+)", text, re.S) if "pq_paged" in k}
    assert spills
    for name, n in spills.items():
        assert n <= (8 if "If" in name else 0), (name, n)
