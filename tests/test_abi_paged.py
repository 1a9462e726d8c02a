"""libembpaged.so loads, exports exactly what include/emb_paged.h declares, and rejects invalid arguments before
touching the GPU (CPU only: no call here reaches a launch)."""
import ctypes
import re
import subprocess

import pytest

import paper_2607_02501_gb300 as emb

# Fake device addresses: only ever used in calls that must fail validation.
GB = 1 << 30
ADDR = [0x7f0000000000 + 4 * GB * i for i in range(16)]


@pytest.fixture(scope="module")
def L():
    emb.build()
    return emb.paged_lib()


def _declared():
    with open(emb.PAGED_HEADER_PATH) as fh:
        return re.findall(r"EMB_API\s+[\w\s\*]*?\b(emb_\w+)\s*\(", fh.read())


def test_exports_are_the_declarations(L):
    out = subprocess.run(["nm", "-D", "--defined-only", emb.PAGED_LIB_PATH], capture_output=True, text=True, check=True).stdout
    assert {line.split()[-1] for line in out.splitlines() if " T " in line} == set(_declared())


def test_workspace_constant_is_the_header_s():
    with open(emb.PAGED_HEADER_PATH) as fh:
        m = re.search(r"#define EMB_PAGED_WORKSPACE \(\(size_t\)(\d+) << (\d+)\)", fh.read())
    assert int(m.group(1)) << int(m.group(2)) == emb.EMB_PAGED_WORKSPACE


def _call(fn, good, change):
    args = dict(good)
    args.update(change)
    return fn(*args.values())


SLOTS = dict(cached=ADDR[0], added=ADDR[1], n_req=4, free=ADDR[2], n_free=10, used=ADDR[3], page=16, table=ADDR[4],
             max_pages=8, q_start=ADDR[5], kv_len=ADDR[6], slots=ADDR[7], positions=ADDR[8], n_tokens=20, used_out=ADDR[9],
             stream=None)


@pytest.mark.parametrize("change,want", [
    ({"n_req": 0}, "EINVAL"), ({"n_req": 65537}, "EINVAL"), ({"n_tokens": -1}, "EINVAL"), ({"n_tokens": 1 << 31}, "EINVAL"),
    ({"page": 0}, "EINVAL"), ({"page": 65537}, "EINVAL"), ({"max_pages": 0}, "EINVAL"), ({"n_free": -1}, "EINVAL"),
    ({"cached": None}, "EINVAL"), ({"added": None}, "EINVAL"), ({"used": None}, "EINVAL"), ({"table": None}, "EINVAL"),
    ({"free": None}, "EINVAL"), ({"slots": None}, "EINVAL"), ({"positions": None}, "EINVAL"), ({"used_out": None}, "EINVAL"),
    ({"q_start": None}, "EINVAL"), ({"kv_len": None}, "EINVAL"),
    ({"slots": ADDR[7] + 4}, "EALIGN"), ({"cached": ADDR[0] + 2}, "EALIGN"), ({"used_out": ADDR[9] + 1}, "EALIGN"),
    ({"used_out": ADDR[3]}, "EINVAL"), ({"kv_len": ADDR[0] + 8}, "EINVAL"), ({"q_start": ADDR[4] + 64}, "EINVAL"),
    ({"positions": ADDR[7] + 80}, "EINVAL"), ({"table": ADDR[2]}, "EINVAL")])
def test_slots_rejects(L, change, want):
    assert _call(L.emb_paged_slots, SLOTS, change) == getattr(emb, "EMB_" + want)


QK = dict(q=ADDR[0], qs=1024, k=ADDR[1], ks=128, v=ADDR[2], vs=128, T=10, H=8, Hk=1, d=128, qg=ADDR[3], kg=ADDR[4], eps=1e-6,
          positions=ADDR[5], pos_stride=10, axes=2, axis=bytes([0, 1] * 32), rot=128, base=1e4, slots=ADDR[6], out=ADDR[7],
          kc=ADDR[8], vc=ADDR[9], n_pages=5, page=16, stream=None)


@pytest.mark.parametrize("change,want", [
    ({"T": 0}, "EINVAL"), ({"H": 0}, "EINVAL"), ({"H": 4097}, "EINVAL"), ({"Hk": 0}, "EINVAL"), ({"d": 12}, "EINVAL"),
    ({"d": 264, "qs": 8 * 264, "ks": 264, "vs": 264}, "EINVAL"), ({"rot": 136}, "EINVAL"), ({"rot": 4}, "EINVAL"),
    ({"rot": -8}, "EINVAL"), ({"axes": 0}, "EINVAL"), ({"axes": 5}, "EINVAL"), ({"axes": 1}, "EINVAL"),
    ({"axis": bytes([2] * 64)}, "EINVAL"), ({"pos_stride": 9}, "EINVAL"), ({"qs": 1016}, "EINVAL"), ({"ks": 130}, "EINVAL"),
    ({"vs": 120}, "EINVAL"), ({"eps": -1.0}, "EINVAL"), ({"eps": float("nan")}, "EINVAL"), ({"base": 0.0}, "EINVAL"),
    ({"base": float("inf")}, "EINVAL"), ({"n_pages": 0}, "EINVAL"), ({"page": 0}, "EINVAL"),
    ({"q": None}, "EINVAL"), ({"k": None}, "EINVAL"), ({"v": None}, "EINVAL"), ({"positions": None}, "EINVAL"),
    ({"slots": None}, "EINVAL"), ({"out": None}, "EINVAL"), ({"kc": None}, "EINVAL"), ({"vc": None}, "EINVAL"),
    ({"q": ADDR[0] + 8}, "EALIGN"), ({"kg": ADDR[4] + 4}, "EALIGN"), ({"vc": ADDR[9] + 2}, "EALIGN"),
    ({"positions": ADDR[5] + 2}, "EALIGN"), ({"slots": ADDR[6] + 4}, "EALIGN"),
    ({"out": ADDR[0]}, "EINVAL"), ({"vc": ADDR[8] + 256}, "EINVAL"), ({"kc": ADDR[1] + 1024}, "EINVAL"),
    ({"out": ADDR[6] + 16}, "EINVAL")])
def test_qk_norm_rope_rejects(L, change, want):
    assert _call(L.emb_qk_norm_rope, QK, change) == getattr(emb, "EMB_" + want)


ATTN = dict(Q=ADDR[0], kc=ADDR[1], vc=ADDR[2], n_pages=40, page=16, table=ADDR[3], max_pages=10, q_start=ADDR[4], kv=ADDR[5],
            prefix=ADDR[6], n_req=3, T=20, max_q=10, O=ADDR[7], H=8, Hk=2, d=128, scale=0.1, cap=0.0, window=0, ws=ADDR[8],
            ws_bytes=emb.EMB_PAGED_WORKSPACE, stream=None)


@pytest.mark.parametrize("change,want", [
    ({"n_req": 0}, "EINVAL"), ({"n_req": 65537}, "EINVAL"), ({"T": 0}, "EINVAL"), ({"max_q": 0}, "EINVAL"), ({"H": 9}, "EINVAL"),
    ({"Hk": 0}, "EINVAL"), ({"H": 8192}, "EINVAL"), ({"scale": float("nan")}, "EINVAL"), ({"cap": -1.0}, "EINVAL"),
    ({"cap": float("inf")}, "EINVAL"), ({"window": -1}, "EINVAL"), ({"n_pages": 0}, "EINVAL"), ({"max_pages": 0}, "EINVAL"),
    ({"Q": None}, "EINVAL"), ({"kc": None}, "EINVAL"), ({"vc": None}, "EINVAL"), ({"table": None}, "EINVAL"),
    ({"q_start": None}, "EINVAL"), ({"kv": None}, "EINVAL"), ({"O": None}, "EINVAL"), ({"ws": None}, "EINVAL"),
    ({"d": 96}, "EUNSUPPORTED"), ({"page": 8}, "EUNSUPPORTED"), ({"page": 48}, "EUNSUPPORTED"), ({"page": 512}, "EUNSUPPORTED"),
    ({"H": 130}, "EUNSUPPORTED"), ({"max_pages": 1 << 27, "n_req": 1}, "EINVAL"),
    ({"max_pages": 1 << 26, "T": 1 << 20, "n_req": 1}, "EUNSUPPORTED"),
    ({"Q": ADDR[0] + 8}, "EALIGN"), ({"O": ADDR[7] + 2}, "EALIGN"), ({"table": ADDR[3] + 2}, "EALIGN"), ({"ws": ADDR[8] + 16}, "EALIGN"),
    ({"prefix": ADDR[6] + 1}, "EALIGN"), ({"ws_bytes": emb.EMB_PAGED_WORKSPACE - 1}, "ENOSPC"),
    ({"O": ADDR[0]}, "EINVAL"), ({"O": ADDR[2] + 1024}, "EINVAL"), ({"ws": ADDR[1]}, "EINVAL"), ({"ws": ADDR[7]}, "EINVAL")])
def test_attention_rejects(L, change, want):
    assert _call(L.emb_paged_attention, ATTN, change) == getattr(emb, "EMB_" + want)


def test_axis_list_of_the_wrong_length_is_refused(L):
    import torch
    t = torch.zeros(1, 128, dtype=torch.bfloat16)
    cache = torch.zeros(1, 16, 1, 128, dtype=torch.bfloat16)
    with pytest.raises(emb.EmbError):
        emb.emb_qk_norm_rope(t, t, t, t, cache, cache, torch.zeros(1, dtype=torch.int64), torch.zeros(1, dtype=torch.int32),
                             axis_of_pair=[0] * 63, stream=1)


def test_binding_reads_its_arguments(L):
    """A wrong number of dimensions is a Python error; what the library refuses raises EmbError."""
    import torch
    i32, cache = torch.zeros(2, dtype=torch.int32), torch.zeros(1, 16, 1, 64, dtype=torch.bfloat16)
    q = torch.zeros(2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        emb.emb_paged_attention(q, cache[0], cache, i32[None], i32, i32, q, 0.1, 1, torch.zeros(16, dtype=torch.uint8), stream=1)
    with pytest.raises(AttributeError):
        emb.emb_paged_slots(None, i32, i32, i32, None, i32, i32, i32, i32, i32, 16, stream=1)
    with pytest.raises(emb.EmbError) as e:
        emb.emb_paged_attention(q, cache, cache, i32[None], i32, i32[:1], torch.empty_like(q), 0.1, 1, torch.zeros(16, dtype=torch.uint8), stream=1)
    assert e.value.status in (emb.EMB_ENOSPC, emb.EMB_EALIGN)
    with pytest.raises(emb.EmbError):
        emb.emb_paged_slots(i32, i32, i32, i32[:1], i32[:, None], i32, i32, i32.long(), i32, i32[:1], 0, stream=1)


def test_declarations_cite_their_passage():
    with open(emb.PAGED_HEADER_PATH) as fh:
        text = fh.read()
    body, prev = text[text.index('extern "C" {'):], 0
    for d in re.finditer(r"EMB_API\s+[\w\s\*]*?\b(emb_\w+)\s*\(", body):
        comments = re.findall(r"/\*.*?\*/", body[prev:d.start()], flags=re.S)
        assert comments and re.search(r"\bSection\s+\d", comments[-1]), d.group(1)
        prev = body.index(";", d.end()) + 1
