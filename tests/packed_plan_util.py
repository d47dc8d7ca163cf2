"""The plan of the packed attention (which tiles, key ranges and scratch rows its work items have) run on the CPU from the kernel's own text, and
what must hold for every plan: the attention and join kernels read and write where it says, without checks of their own."""
import ctypes
import os
import re
import subprocess
import tempfile

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2503_14985_b200", "csrc")
GUARD = 4096
_lib = None


def _cut(text, first, last):
    a = text.index(first)
    return text[a: text.index(last, a)]


def plan_source():
    packed = open(os.path.join(CSRC, "mha_packed.cuh")).read()
    calls = open(os.path.join(CSRC, "mlt.cu")).read()
    text = _cut(packed, "constexpr unsigned int kStatusBadSequence", "constexpr int kPackedPlanSmem")
    text = re.sub(r"extern __shared__ int4 plan_smem\[\];", "int4* plan_smem = reinterpret_cast<int4*>(plan_memory);", text)
    text += re.search(r"constexpr int kPackedPlanSmem[^;]*;", packed).group(0) + "\nstatic_assert(kPackedPlanSmem <= sizeof(plan_memory), \"\");\n"
    text += _cut(packed, "struct PackedScratch", "inline int packed_configure")
    text += _cut(calls, "int64_t packed_part_limit", "int packed_cache_maps")
    return text


def load():
    global _lib
    if _lib is None:
        source = plan_source()
        host = os.path.join(HERE, "packed_plan_host.cpp")
        with tempfile.TemporaryDirectory(prefix="packed_plan_") as folder:
            with open(os.path.join(folder, "packed_plan_source.inc"), "w") as f:
                f.write(source)
            out = os.path.join(folder, "plan.so")
            # (_FORTIFY_SOURCE takes a jump to another stack for an error)
            res = subprocess.run(["g++", "-std=c++17", "-O2", "-U_FORTIFY_SOURCE", "-w", "-shared", "-fPIC", "-I", folder, "-o", out, host], capture_output=True,
                                 text=True)
            assert res.returncode == 0, res.stderr
            _lib = ctypes.CDLL(out)
        _lib.packed_scratch_layout.restype = ctypes.c_longlong
    return _lib


def _ptr(a):
    return None if a is None else a.ctypes.data_as(ctypes.c_void_p)


KINDS = {"packed": 0, "prefill": 1, "shared": 2}


def plan(kind, T, cu_q, G, Hk, D, cu_k=None, num_k=0, context=None, prefix=None, lens=None, causal=True, bs=16, max_blocks=0, sms=148, parts=None):
    """The plan of a call, checked.  parts: rows of partial results that the scratch has room for (default: all).  Returns a dict."""
    lib = load()
    i32 = [None if a is None else np.ascontiguousarray(a, np.int32) for a in (cu_q, cu_k, context, prefix, lens)]
    S = len(i32[0]) - 1
    names = ("seqs", "key_base", "entries", "entry_rows", "tile_info", "lists", "row_bytes", "part_rows", "max_tiles", "max_entries", "W")
    raw = (ctypes.c_longlong * len(names))()
    lib.packed_scratch_layout(KINDS[kind], ctypes.c_longlong(T), ctypes.c_longlong(S), G, Hk, D, raw)
    x = dict(zip(names, raw))
    size = x["lists"] + (x["part_rows"] if parts is None else parts) * x["row_bytes"]
    # (the plan writes the lists only: what follows them stands for the partial results and what lies behind the scratch)
    buf = np.full(x["lists"] + GUARD, 0xAB, np.uint8)
    status, rows = np.zeros(4, np.uint32), ctypes.c_int()
    rc = lib.run_packed_plan(KINDS[kind], T, S, num_k, G, Hk, D, int(causal), bs, max_blocks, sms, *[_ptr(a) for a in i32], _ptr(buf), ctypes.c_longlong(size),
                             ctypes.byref(rows), _ptr(status))
    assert rc == 0, "threads that do not meet at a barrier"
    assert (buf[x["lists"]:] == 0xAB).all(), "written behind the lists"
    n_all = S + T if kind == "shared" else S
    items, _, chunk, _ = buf[:16].view(np.int32)
    assert items % Hk == 0
    entries = items // Hk
    assert 0 <= entries <= x["max_entries"], "more entries than the list holds"
    at = buf.ctypes.data
    seqs = np.frombuffer((ctypes.c_char * (16 * n_all)).from_address(at + x["seqs"]), np.int32).reshape(-1, 4).copy()
    e = np.frombuffer((ctypes.c_char * (16 * entries)).from_address(at + x["entries"]), np.int32).reshape(-1, 4).copy() if entries else np.zeros((0, 4), np.int32)
    e_rows = np.frombuffer((ctypes.c_char * (4 * entries)).from_address(at + x["entry_rows"]), np.int32).copy() if entries else np.zeros(0, np.int32)
    info = buf[x["tile_info"]: x["lists"]].view(np.int32)
    info = info[: len(info) // 2 * 2].reshape(-1, 2)
    W, W2 = x["W"], 2 * x["W"]
    part_rows = rows.value
    covered, taken = {}, []
    for (s, pair, b0, nb), row in zip(e.tolist(), e_rows.tolist()):
        assert 0 <= s < n_all, "an entry of no sequence"
        first, tokens, keys, before = seqs[s].tolist()
        n = min(W2, tokens - pair * W2)
        assert pair >= 0 and n > 0, "an entry without tokens"
        limit = T if s < S else s - S + 1
        assert 0 <= first and first + tokens <= limit, "tokens beyond the call's"
        last = keys - tokens + pair * W2 + n if (causal and kind != "shared") else keys
        blocks = -(-max(0, last) // 128)
        assert 0 <= b0 and 0 <= nb and b0 + nb <= blocks, "key blocks beyond the sequence's"
        covered.setdefault((s, pair), []).append((b0, nb))
        uses_parts = part_rows > 0 and chunk > 0 and (kind == "shared" or n <= W or blocks > chunk)
        if uses_parts:
            each = 2 * n * G if n <= W else 256
            for h in range(Hk):
                taken.append((row + h * each, row + (h + 1) * each))
            a = before + pair
            assert 0 <= a < len(info) and row == info[a, 0] + (b0 // chunk) * each * Hk, "the join looks for the part elsewhere"
    for (s, pair), ranges in covered.items():
        first, tokens, keys, before = seqs[s].tolist()
        n = min(W2, tokens - pair * W2)
        last = keys - tokens + pair * W2 + n if (causal and kind != "shared") else keys
        blocks = -(-max(0, last) // 128)
        ranges.sort()
        assert ranges[0][0] == 0 and sum(r[1] for r in ranges) == blocks, "key blocks left out"
        assert all(a[0] + a[1] == b[0] for a, b in zip(ranges, ranges[1:])), "key blocks twice or not at all"
        if chunk > 0 and part_rows > 0:
            assert info[before + pair, 1] == len(ranges), "the join takes another number of parts"
    taken.sort()
    assert all(a[1] <= b[0] for a, b in zip(taken, taken[1:])), "two parts in the same rows"
    assert not taken or (taken[0][0] >= 0 and taken[-1][1] <= part_rows), f"parts in rows {taken[0][0]} .. {taken[-1][1]} of {part_rows}"
    if entries:  # every tile of every sequence that is not left out
        assert len(covered) == sum(-(-t // W2) for t in seqs[:, 1].tolist()), "tiles left out or twice"
    return dict(x, status=int(status[0]), chunk=int(chunk), entries=e, seqs=seqs, part_rows=part_rows, top=taken[-1][1] if taken else 0, num=int(entries))
