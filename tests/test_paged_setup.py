"""What a paged call asks of the CUDA runtime beside its launch, against one that counts (tests/fake_paged_cuda.cpp).  Needs no GPU."""
import ctypes
import os
import subprocess

import pytest

from paper_2604_24432_b200 import binding as ksa
from paper_2604_24432_b200 import build as ksa_build
from tests.test_schedule_memory import _run, _symbols

HERE = os.path.dirname(os.path.abspath(__file__))


class Counts(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("properties", "attributes", "launches", "maps")]


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    ksa_build.build()
    d = str(tmp_path_factory.mktemp("fake"))
    hosts = [os.path.join(ksa_build.OBJ_DIR, n) for n in ("ksa_api.o", "ksa_paged.o", "ksa_paged_attn.o", "ksa_paged_tc.o")]
    obj, lib = os.path.join(d, "fake.o"), os.path.join(d, "libfake.so")
    cuda = os.path.join(os.path.dirname(os.path.dirname(ksa_build._nvcc())) or "/usr/local/cuda", "include")
    _run("g++", "-std=c++17", "-O1", "-fPIC", "-I" + cuda, "-c", os.path.join(HERE, "fake_paged_cuda.cpp"), "-o", obj)
    missing = set().union(*(_symbols(o, "-u") for o in hosts + [obj])) - set().union(*(_symbols(o, "--defined-only") for o in hosts + [obj]))
    missing = sorted(s for s in missing if s.startswith(("cuda", "__cuda", "_ZN3ksa")))
    with open(os.path.join(d, "stubs.s"), "w") as f:
        f.write(".text\n" + "".join(".globl %s\n.type %s, @function\n%s:\n" % (s, s, s) for s in missing) + "xorl %eax, %eax\nret\n.section .note.GNU-stack,\"\",@progbits\n")
    _run("g++", "-shared", "-fPIC", "-Wl,-Bsymbolic", "-o", lib, *hosts, obj, os.path.join(d, "stubs.s"))
    L = ctypes.CDLL(lib)
    L.fake_counts.restype = Counts
    L.ksa_paged_attn.argtypes = [ctypes.c_void_p] * 6 + [ctypes.c_size_t] + [ctypes.c_void_p] * 2
    L.ksa_destroy.argtypes = [ctypes.c_void_p]
    return L


class Context:
    def __init__(self, L, device=0):
        self.L, self.handle = L, ctypes.c_void_p()
        assert L.ksa_create(ctypes.byref(self.handle), device) == ksa.KSA_OK

    def attn(self, rows=1, **other):
        D, Hkv, ps = 128, 2, 64
        p = ksa.ksa_paged_params(struct_size=ctypes.sizeof(ksa.ksa_paged_params), batch=1, num_rows=rows, chunk_len=8, summaries_per_chunk=1, window_chunks=4,
                                 num_q_heads=8, num_kv_heads=Hkv, head_dim=D, softmax_scale=0.1, flags=0, kv_format=ksa.KSA_KV_BF16, page_rows=ps,
                                 num_pages=7, text_cols=30, summ_cols=4, page_stride=Hkv * ps * D, head_stride=ps * D, row_stride=D,
                                 q_stride_tok=8 * D, q_stride_head=D, o_stride_tok=8 * D, o_stride_head=D)
        kv = ksa.ksa_paged_kv(**{**{n: 0x10000 * (i + 1) for i, (n, _) in enumerate(ksa.ksa_paged_kv._fields_)}, **other})
        return self.L.ksa_paged_attn(self.handle, ctypes.addressof(kv), 0x900000, 0xA00000, 0xB00000, None, 0, ctypes.addressof(p), None)

    def close(self):
        self.L.ksa_destroy(self.handle)


def _spent(L, f):
    before = L.fake_counts()
    f()
    after = L.fake_counts()
    return {n: getattr(after, n) - getattr(before, n) for n, _ in Counts._fields_}


def test_a_device_is_asked_and_set_up_once(fake):
    first = Context(fake)
    assert _spent(fake, first.attn)["attributes"] == 20             # a shared-memory opt-in a kernel
    assert _spent(fake, first.attn) == dict(properties=0, attributes=0, launches=1, maps=2)
    made = []
    assert _spent(fake, lambda: made.append(Context(fake))) == dict(properties=0, attributes=0, launches=0, maps=0)
    assert _spent(fake, lambda: made[0].attn(500)) == dict(properties=0, attributes=0, launches=1, maps=2)
    first.close()
    assert _spent(fake, made[0].attn)["attributes"] == 0
    other = Context(fake, 1)                                         # a device of its own
    assert _spent(fake, other.attn)["attributes"] == 20
    other.close(), made[0].close()
    again = Context(fake)                                            # (the device may have been reset when nobody held it)
    assert _spent(fake, again.attn)["attributes"] == 20
    again.close()


def test_a_setup_that_fails_is_tried_again(fake):
    c = Context(fake)
    fake.fake_fail_attribute(3)
    assert c.attn() == ksa.KSA_ERR_CUDA
    assert c.attn() == ksa.KSA_OK and _spent(fake, c.attn)["attributes"] == 0
    c.close()


@pytest.mark.parametrize("name", ["text_table", "summ_table", "cached", "cu_rows"])
def test_integers_out_of_alignment_are_refused(fake, name):
    c = Context(fake)
    for off in (1, 2, 3):
        assert c.attn(**{name: 0x40000 + off}) == ksa.KSA_ERR_INVALID_ARG
    assert c.attn(**{name: 0x40004}) == ksa.KSA_OK
    c.close()
