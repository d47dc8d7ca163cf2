"""The BF16 serving path without a GPU: what its Python entry points refuse, and that its kernels, which are launched while the kernel before
them in the stream may still run, touch no device memory before their wait."""
import os
import re

import pytest

torch = pytest.importorskip("torch")

import paper_2503_14985_b200 as mlt  # noqa: E402
from test_f8_launch_order import WAIT, block, source  # noqa: E402

BF, I32 = torch.bfloat16, torch.int32
KERNELS = [(name, m.group(1), block(source(name), m.end())) for name in ("mha_packed.cuh", "gemm_w4.cuh")
           for m in re.finditer(r"__global__[^;{]*?(\w+_kernel)\s*\(", source(name))]


def test_every_kernel_is_seen():
    assert {k for _, k, _ in KERNELS} == {"mha_packed_plan_kernel", "mha_packed_kernel", "mha_packed_join_kernel", "gemm_w4_kernel"}


@pytest.mark.parametrize("name,kernel,body", KERNELS, ids=[k for _, k, _ in KERNELS])
def test_nothing_is_touched_before_the_wait(name, kernel, body):
    wait = WAIT.search(body)
    assert wait, "the kernel does not wait"
    before = body[:wait.start()]
    pointers = set()
    for m in re.finditer(r"\bstruct \w+Params\b", source(name)):
        for decl in block(source(name), m.end()).split(";"):
            if "*" in decl:
                pointers |= set(re.findall(r"\w+", decl.split("*", 1)[1]))
    assert pointers and not re.search(r"\bp\.(%s)\b" % "|".join(sorted(pointers)), before)
    assert not re.search(r"[(,]\s*p\s*[,)]", before), "the parameters go to a function before the wait"
    assert not re.search(r"\bclock_probe\b|\bg_status\b|\bpacked_report\b|\bst\.global\b|\btma_load|\btma_store_[23]d", before)
    assert not re.search(r"\b__ldg\b|\bld\.global\.nc\b|\b__restrict__\b", source(name))
    # every CTA waits: none may end before the kernels in front of its own have
    assert not re.search(r"\breturn;", before)


def packed_args():
    x = torch.zeros(5, 4, 64, dtype=BF)
    return [x, x[:, :2].contiguous(), x[:, :2].contiguous(), torch.zeros(3, dtype=I32), torch.zeros(3, dtype=I32)]


def paged_args():
    q, cache = torch.zeros(2, 4, 64, dtype=BF), torch.zeros(5, 2, 16, 64, dtype=BF)
    return [q, cache, cache]


@pytest.mark.parametrize("change,error,match", [
    (lambda a: a.__setitem__(0, a[0].float()), TypeError, "bfloat16"), (lambda a: a.__setitem__(0, a[0].view(5, 256)), TypeError, "heads"),
    (lambda a: a.__setitem__(1, a[1][:, :, :32]), ValueError, "shape"), (lambda a: a.__setitem__(2, a[2][:4]), ValueError, "shape"),
    (lambda a: a.__setitem__(3, a[3].long()), TypeError, "int32"), (lambda a: a.__setitem__(4, a[4][:2]), ValueError, "cu_q"),
    (lambda a: a.__setitem__(0, a[0].transpose(0, 1).contiguous().transpose(0, 1)), ValueError, "side by side"),
    (lambda a: a.__setitem__(3, torch.zeros(6, dtype=I32)[::2]), TypeError, "contiguous"), (lambda a: None, ValueError, "CUDA")])
def test_packed_wrapper(change, error, match):
    a = packed_args()
    change(a)
    with pytest.raises(error, match=match):
        mlt.mha_packed_fwd(*a, causal=True, scale=0.1)


def test_outputs_and_scratch_of_the_wrong_kind():
    a = packed_args()
    for kw, error in ((dict(O=torch.zeros(5, 4, 64)), ValueError), (dict(O=torch.zeros(5, 4, 32, dtype=BF)), ValueError),
                      (dict(LSE=torch.zeros(4, 5)), ValueError), (dict(LSE=torch.zeros(5, 4, dtype=BF)), ValueError),
                      (dict(LSE=torch.zeros(4, 5).t()), ValueError), (dict(workspace=torch.zeros(1 << 20, dtype=torch.uint8)[::2]), TypeError)):
        with pytest.raises(error):
            mlt.mha_packed_fwd(*a, causal=True, scale=0.1, **kw)


def test_prefill_and_shared_wrappers():
    q, kc, vc = paged_args()
    cu, ctx, table, lens = torch.zeros(3, dtype=I32), torch.zeros(2, dtype=I32), torch.zeros(2, 3, dtype=I32), torch.zeros(2, dtype=I32)
    for args in ((q.float(), kc, vc, cu, ctx, table), (q, kc.float(), vc, cu, ctx, table), (q, kc, vc, cu.long(), ctx, table),
                 (q, kc.transpose(1, 2), vc, cu, ctx, table)):
        with pytest.raises(TypeError):
            mlt.paged_attn_prefill(*args, scale=0.1)
    for args in ((q, kc, vc[:4], cu, ctx, table), (q, kc, vc, cu[:2], ctx, table), (q, kc, vc, cu, ctx, table[:1]), (q, kc, vc, cu, ctx, table[0]),
                 (q[:, :, :32].contiguous(), kc, vc, cu, ctx, table), (q, kc, vc, cu, ctx, table)):
        with pytest.raises(ValueError):
            mlt.paged_attn_prefill(*args, scale=0.1)
    prefix, groups = torch.zeros(1, dtype=I32), torch.zeros(2, dtype=I32)
    for args in ((q.transpose(0, 1), kc, vc, table, lens, prefix, groups), (q, kc, vc, table, lens.long(), prefix, groups)):
        with pytest.raises(TypeError):
            mlt.paged_attn_decode_shared(*args, scale=0.1)
    for args in ((q, kc, vc, table, lens, prefix, groups[:1]), (q, kc, vc, table[:1], lens, prefix, groups), (q, kc, vc, table, lens[:1], prefix, groups),
                 (q, kc, vc[:2], table, lens, prefix, groups), (q, kc, vc, table, lens, prefix, groups)):
        with pytest.raises(ValueError):
            mlt.paged_attn_decode_shared(*args, scale=0.1)
    with pytest.raises(ValueError):
        mlt.paged_attn_decode_shared(q, kc, vc, table, lens, prefix, groups, scale=0.1, O=torch.zeros(2, 8, 64, dtype=BF)[:, ::2])


def test_w4_wrapper():
    x, w, s, z = torch.zeros(2, 256, dtype=BF), torch.zeros(9, 128, dtype=torch.uint8), torch.zeros(9, 4, dtype=BF), torch.zeros(9, 4, dtype=torch.uint8)
    for args in ((x.float(), w, s, z), (x, w.to(torch.int8), s, z), (x, w, s.float(), z), (x, w, s, z.to(I32))):
        with pytest.raises(TypeError):
            mlt.gemm_w4(*args)
    for args in ((x[:, :128], w, s, z), (x, w[:8], s, z), (x, w, s, z[:8]), (x, w, s[:, :3], z[:, :3]), (x, w.t().contiguous().t(), s, z), (x, w, s, z)):
        with pytest.raises(ValueError):
            mlt.gemm_w4(*args)
    for s2 in (torch.zeros(9, 2, dtype=BF), torch.zeros(9, 16, dtype=BF)):
        with pytest.raises((ValueError, mlt.MltError)):
            mlt.gemm_w4(x, w, s2)
    with pytest.raises(ValueError):
        mlt.gemm_w4(x, w, s, z, torch.zeros(2, 8, dtype=BF))
