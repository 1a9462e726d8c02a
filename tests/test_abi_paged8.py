"""The 8-bit cache's entry points reject invalid arguments before touching the GPU, and tensors that are not what the call would take
them for (CPU only: no call here reaches a launch)."""
import pytest
import torch

import paper_2607_02501_gb300 as emb

GB = 1 << 30
ADDR = [0x7f0000000000 + 4 * GB * i for i in range(24)]  # fake device addresses


@pytest.fixture(scope="module", autouse=True)
def L():
    emb.build()
    return emb.paged_lib()


def _call(fn, good, change):
    args = dict(good)
    args.update(change)
    return fn(*args.values())


STORE = dict(q=ADDR[0], q_stride=1024, k=ADDR[1], k_stride=256, v=ADDR[2], v_stride=256, n_tokens=20, n_heads=8, n_kv_heads=2, head_dim=128,
             q_gamma=ADDR[3], k_gamma=ADDR[4], eps=1e-6, positions=ADDR[5], pos_stride=20, n_axes=1, axis=None, turns=ADDR[6], rot_dim=128,
             neighbours=0, factor=1.0, slots=ADDR[7], q_out=ADDR[8], k_codes=ADDR[9], v_codes=ADDR[10], k_exp=ADDR[11], v_exp=ADDR[12],
             n_pages=4, page_size=16, stream=None)


@pytest.mark.parametrize("change,want", [
    ({"n_tokens": 0}, "EINVAL"), ({"n_tokens": 1 << 31}, "EINVAL"), ({"n_heads": 0}, "EINVAL"), ({"n_heads": 4097}, "EINVAL"),
    ({"n_kv_heads": 0}, "EINVAL"), ({"head_dim": 0}, "EINVAL"), ({"head_dim": 96}, "EUNSUPPORTED"), ({"head_dim": 512}, "EUNSUPPORTED"),
    ({"page_size": 0}, "EINVAL"), ({"page_size": 8}, "EUNSUPPORTED"), ({"page_size": 48}, "EUNSUPPORTED"), ({"page_size": 512}, "EUNSUPPORTED"),
    ({"n_pages": 0}, "EINVAL"), ({"n_pages": 1 << 31}, "EINVAL"), ({"rot_dim": -8}, "EINVAL"), ({"rot_dim": 136}, "EINVAL"),
    ({"rot_dim": 60}, "EINVAL"), ({"n_axes": 0}, "EINVAL"), ({"n_axes": 5}, "EINVAL"), ({"pos_stride": 19}, "EINVAL"),
    ({"eps": -1.0}, "EINVAL"), ({"eps": float("nan")}, "EINVAL"), ({"factor": float("inf")}, "EINVAL"), ({"neighbours": 2}, "EINVAL"),
    ({"q_stride": 1016}, "EINVAL"), ({"k_stride": 260}, "EINVAL"), ({"v_stride": 248}, "EINVAL"), ({"q_stride": 1 << 45}, "EINVAL"),
    ({"turns": None}, "EINVAL"), ({"q": None}, "EINVAL"), ({"k": None}, "EINVAL"), ({"v": None}, "EINVAL"), ({"positions": None}, "EINVAL"),
    ({"slots": None}, "EINVAL"), ({"q_out": None}, "EINVAL"), ({"k_codes": None}, "EINVAL"), ({"v_codes": None}, "EINVAL"),
    ({"k_exp": None}, "EINVAL"), ({"v_exp": None}, "EINVAL"),
    ({"q": ADDR[0] + 8}, "EALIGN"), ({"k": ADDR[1] + 2}, "EALIGN"), ({"v_codes": ADDR[10] + 8}, "EALIGN"), ({"q_out": ADDR[8] + 8}, "EALIGN"),
    ({"q_gamma": ADDR[3] + 4}, "EALIGN"), ({"positions": ADDR[5] + 2}, "EALIGN"), ({"slots": ADDR[7] + 4}, "EALIGN"),
    ({"turns": ADDR[6] + 4}, "EALIGN"),
    ({"q_out": ADDR[0]}, "EINVAL"), ({"v_codes": ADDR[9] + 16}, "EINVAL"), ({"v_exp": ADDR[11] + 7}, "EINVAL"), ({"k_exp": ADDR[9] + 64}, "EINVAL"),
    ({"k_codes": ADDR[1]}, "EINVAL"), ({"v_exp": ADDR[7]}, "EINVAL"), ({"k_exp": ADDR[6] + 500}, "EINVAL"),
    ({"n_tokens": 1 << 30, "n_heads": 4096, "q_stride": 1 << 15, "head_dim": 64, "q": 1 << 52, "pos_stride": 1 << 30, "rot_dim": 64}, "EINVAL"),
    ({"n_tokens": (1 << 31) - 1, "pos_stride": 1 << 31, "n_heads": 8, "head_dim": 64, "rot_dim": 0, "q_stride": 512, "n_kv_heads": 2,
      "k_stride": 128, "v_stride": 128}, "EUNSUPPORTED")])
def test_store_rejects(L, change, want):
    assert _call(L.emb_paged8_store, STORE, change) == getattr(emb, "EMB_" + want)


READ = dict(k_codes=ADDR[0], v_codes=ADDR[1], k_exp=ADDR[2], v_exp=ADDR[3], n_pages=4, page_size=16, n_kv_heads=2, head_dim=64,
            slots=ADDR[4], n_rows=10, k_out=ADDR[5], v_out=ADDR[6], stream=None)


@pytest.mark.parametrize("change,want", [
    ({"n_rows": -1}, "EINVAL"), ({"n_rows": 1 << 31}, "EINVAL"), ({"n_pages": 0}, "EINVAL"), ({"page_size": 24}, "EUNSUPPORTED"),
    ({"head_dim": 32}, "EUNSUPPORTED"), ({"head_dim": -64}, "EINVAL"), ({"n_kv_heads": 4097}, "EINVAL"), ({"slots": None}, "EINVAL"),
    ({"k_out": None}, "EINVAL"), ({"v_out": None}, "EINVAL"), ({"k_codes": None}, "EINVAL"), ({"v_exp": None}, "EINVAL"),
    ({"k_codes": ADDR[0] + 4}, "EALIGN"), ({"v_out": ADDR[6] + 2}, "EALIGN"), ({"slots": ADDR[4] + 2}, "EALIGN"),
    ({"v_out": ADDR[5] + 1024}, "EINVAL"), ({"k_out": ADDR[0]}, "EINVAL"), ({"v_out": ADDR[4]}, "EINVAL"), ({"n_rows": 0, "slots": None}, "OK")])
def test_read_rejects(L, change, want):
    assert _call(L.emb_paged8_read, READ, change) == getattr(emb, "EMB_" + want)


ATTN = dict(Q=ADDR[0], k=ADDR[1], v=ADDR[2], ke=ADDR[3], ve=ADDR[4], n_pages=10, page=16, table=ADDR[5], max_pages=8, q_start=ADDR[6],
            kv_len=ADDR[7], prefix=ADDR[8], n_req=3, n_tokens=20, max_q=4, O=ADDR[9], n_heads=8, n_kv_heads=2, head_dim=128, scale=0.1,
            cap=0.0, window=0, workspace=ADDR[10], ws_bytes=emb.EMB_PAGED_WORKSPACE, stream=None)


@pytest.mark.parametrize("change,want", [
    ({"n_req": 0}, "EINVAL"), ({"n_tokens": 0}, "EINVAL"), ({"max_q": 0}, "EINVAL"), ({"n_heads": 7}, "EINVAL"), ({"n_kv_heads": 0}, "EINVAL"),
    ({"scale": float("nan")}, "EINVAL"), ({"cap": -1.0}, "EINVAL"), ({"window": -1}, "EINVAL"), ({"head_dim": 80}, "EUNSUPPORTED"),
    ({"page": 20}, "EUNSUPPORTED"), ({"page": 0}, "EINVAL"), ({"n_heads": 130}, "EUNSUPPORTED"), ({"ke": None}, "EINVAL"), ({"ve": None}, "EINVAL"),
    ({"k": None}, "EINVAL"), ({"v": None}, "EINVAL"), ({"Q": None}, "EINVAL"), ({"O": None}, "EINVAL"), ({"workspace": None}, "EINVAL"),
    ({"k": ADDR[1] + 8}, "EALIGN"), ({"table": ADDR[5] + 2}, "EALIGN"), ({"workspace": ADDR[10] + 16}, "EALIGN"),
    ({"ws_bytes": 1024}, "ENOSPC"), ({"O": ADDR[0]}, "EINVAL"), ({"O": ADDR[3]}, "EINVAL"), ({"ve": ADDR[9] + 64}, "EINVAL"),
    ({"ke": ADDR[10] + 4096}, "EINVAL"), ({"O": ADDR[1]}, "EINVAL"), ({"n_pages": 1 << 31}, "EINVAL"), ({"max_pages": 1 << 28}, "EINVAL")])
def test_attention_rejects(L, change, want):
    assert _call(L.emb_paged8_attention, ATTN, change) == getattr(emb, "EMB_" + want)


# ------------------------------------------------------------------ tensors
R, T, H, HK, D, PAGES, PAGE, WIDTH = 3, 10, 4, 2, 64, 5, 32, 6


def _t(dtype, *shape):
    return torch.zeros(*shape, dtype=dtype)


def _refused(call, good, name, bad, words):
    args = dict(good)
    args[name] = bad
    with pytest.raises(emb.EmbError, match=words) as e:
        call(**args, stream=1)
    assert e.value.status == emb.EMB_EINVAL


bf, i32, i64, u8 = torch.bfloat16, torch.int32, torch.int64, torch.uint8
CACHE = dict(k_codes=_t(u8, PAGES, PAGE, HK, D), v_codes=_t(u8, PAGES, PAGE, HK, D), k_exp=_t(u8, PAGES, PAGE // 16, HK), v_exp=_t(u8, PAGES, PAGE // 16, HK))
STORE_T = dict(q=_t(bf, T, H * D), k=_t(bf, T, HK * D), v=_t(bf, T, HK * D), q_out=_t(bf, T, H * D), **CACHE, slots=_t(i64, T), positions=_t(i32, T),
               turns=_t(i64, D // 2), q_gamma=torch.ones(D), k_gamma=torch.ones(D), axis_of_pair=_t(u8, D // 2))


@pytest.mark.parametrize("name,bad,words", [
    ("q", _t(bf, T, H * D + 8), "no whole heads"), ("q", _t(bf, H * D, T).T, "do not lie side by side"), ("q", torch.zeros(T, H * D), "elements of 2 bytes"),
    ("k", _t(bf, T - 1, HK * D), "k: fewer rows"), ("v", _t(bf, T, HK * D - D), "v: fewer rows than q, or heads"), ("k", torch.zeros(T, HK * D), "elements of 2 bytes"),
    ("q_out", _t(bf, T - 1, H * D), "q_out has"), ("q_out", _t(bf, T, 2 * H * D)[:, :H * D], "q_out is not contiguous"),
    ("v_codes", _t(u8, PAGES - 1, PAGE, HK, D), "v_codes has"), ("v_codes", _t(bf, PAGES, PAGE, HK, D), "v_codes: elements of 2"),
    ("k_codes", _t(u8, PAGES, HK, PAGE, D).transpose(1, 2), "k_codes is not contiguous"), ("k_exp", _t(u8, PAGES, 1, HK), "k_exp has 10 elements, 20 needed"),
    ("v_exp", _t(u8, PAGES, HK, PAGE // 16).transpose(1, 2), "v_exp is not contiguous"), ("v_exp", _t(i32, PAGES, PAGE // 16, HK), "v_exp: elements of 4"),
    ("slots", _t(i32, T), "slots: elements of 4"), ("slots", _t(i64, T - 1), "slots has"), ("positions", _t(i32, T - 1), "positions has 9"),
    ("positions", _t(i32, 3, T - 1), "positions has 9 columns"), ("positions", _t(i64, T), "positions: elements of 8"),
    ("turns", torch.zeros(D // 2), "turns: elements of 4"), ("turns", _t(i64, D)[::2], "turns is not contiguous"),
    ("q_gamma", torch.ones(D - 1), "q_gamma has"), ("k_gamma", _t(bf, D), "k_gamma: elements of 2"), ("axis_of_pair", _t(u8, D // 2 - 1), "axis_of_pair has"),
    ("axis_of_pair", _t(i32, D // 2), "axis_of_pair: elements of 4")])
def test_store_tensors(name, bad, words):
    _refused(emb.emb_paged8_store, STORE_T, name, bad, words)


READ_T = dict(**CACHE, slots=_t(i64, T), k_out=_t(bf, T, HK * D), v_out=_t(bf, T, HK * D))


@pytest.mark.parametrize("name,bad,words", [
    ("v_codes", _t(u8, PAGES, PAGE, HK - 1, D), "v_codes has"), ("k_exp", _t(u8, PAGES, PAGE // 16), "k_exp has"), ("slots", _t(i32, T), "slots: elements of 4"),
    ("k_out", _t(bf, T - 1, HK * D), "k_out has"), ("v_out", torch.zeros(T, HK * D), "v_out: elements of 4"), ("v_out", _t(bf, T, 2 * HK * D)[:, ::2], "v_out is not")])
def test_read_tensors(name, bad, words):
    _refused(emb.emb_paged8_read, READ_T, name, bad, words)


ATTN_T = dict(Q=_t(bf, T, H * D), **CACHE, table=_t(i32, R, WIDTH), q_start=_t(i32, R + 1), kv_len=_t(i32, R), O=_t(bf, T, H * D), scale=0.1, max_q=4,
              workspace=torch.zeros(emb.EMB_PAGED_WORKSPACE, dtype=torch.uint8), prefix=_t(i32, R))


@pytest.mark.parametrize("name,bad,words", [
    ("Q", _t(bf, T, H * D + 8), "no whole heads"), ("O", _t(bf, T - 1, H * D), "O has"), ("O", torch.zeros(T, H * D), "O: elements of 4"),
    ("k_codes", _t(u8, PAGES, HK, PAGE, D).transpose(1, 2), "k_codes is not contiguous"), ("v_codes", _t(u8, PAGES, PAGE, HK - 1, D), "v_codes has"),
    ("k_exp", _t(u8, PAGES, 1, HK), "k_exp has"), ("v_exp", _t(bf, PAGES, PAGE // 16, HK), "v_exp: elements of 2"), ("table", _t(i64, R, WIDTH), "table: elements of 8"),
    ("q_start", _t(i32, R), "q_start has"), ("kv_len", _t(i32, R, 2)[:, 1], "kv_len is not contiguous"), ("prefix", _t(i32, R - 1), "prefix has")])
def test_attention_tensors(name, bad, words):
    _refused(emb.emb_paged8_attention, ATTN_T, name, bad, words)


def test_kinds_of_errors():
    with pytest.raises(ValueError):
        emb.emb_paged8_read(CACHE["k_codes"][0], *list(CACHE.values())[1:], _t(i64, T), READ_T["k_out"], READ_T["v_out"], stream=1)
    with pytest.raises(AttributeError):
        emb.emb_paged8_store(None, *list(STORE_T.values())[1:], stream=1)
