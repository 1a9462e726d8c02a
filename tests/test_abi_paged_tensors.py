"""The paged-cache calls refuse tensors that are not what the call would take them for: too short, strided, of elements of
another size, or of shapes that do not go together. CPU only: every call here is refused before it reaches the library."""
import pytest
import torch

import paper_2607_02501_gb300 as emb

R, T, H, HK, D, PAGES, PAGE, WIDTH = 3, 10, 4, 2, 64, 5, 16, 6


@pytest.fixture(scope="module", autouse=True)
def built():
    emb.build()


def _i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def _bf(*shape):
    return torch.zeros(*shape, dtype=torch.bfloat16)


def _refused(call, good, name, bad, words):
    args = dict(good)
    args[name] = bad
    with pytest.raises(emb.EmbError, match=words) as e:
        call(**args, stream=1)
    assert e.value.status == emb.EMB_EINVAL


SLOTS = dict(cached=_i32(R), added=_i32(R), free_pages=_i32(7), used=_i32(1), table=_i32(R, WIDTH), q_start=_i32(R + 1), kv_len=_i32(R),
             slots=torch.zeros(T, dtype=torch.int64), positions=_i32(T), used_out=_i32(1), page_size=PAGE)


@pytest.mark.parametrize("name,bad,words", [
    ("table", _i32(R, WIDTH + 3)[:, :WIDTH], "table is not contiguous"), ("table", _i32(WIDTH, R).T, "table is not contiguous"),
    ("cached", _i32(R - 1), "cached has 2 elements, 3 needed"), ("added", _i32(R - 1), "added has"), ("kv_len", _i32(R - 1), "kv_len has"),
    ("q_start", _i32(R), "q_start has 3 elements, 4 needed"), ("positions", _i32(T - 1), "positions has"), ("used", _i32(0), "used has"),
    ("used_out", _i32(0), "used_out has"), ("cached", _i32(R, 2)[:, 0], "cached is not contiguous"),
    ("slots", torch.zeros(T, 2, dtype=torch.int64)[:, 1], "slots is not contiguous"), ("slots", _i32(T), "slots: elements of 4 bytes, 8 expected"),
    ("positions", torch.zeros(T, dtype=torch.int64), "positions: elements of 8 bytes, 4 expected"),
    ("free_pages", torch.zeros(7, dtype=torch.int64), "free_pages: elements of 8"), ("table", torch.zeros(R, WIDTH, dtype=torch.int64), "table: elements of 8")])
def test_slots(name, bad, words):
    _refused(emb.emb_paged_slots, SLOTS, name, bad, words)


QK = dict(q=_bf(T, H * D), k=_bf(T, HK * D), v=_bf(T, HK * D), q_out=_bf(T, H * D), k_cache=_bf(PAGES, PAGE, HK, D),
          v_cache=_bf(PAGES, PAGE, HK, D), slots=torch.zeros(T, dtype=torch.int64), positions=_i32(T), q_gamma=torch.ones(D), k_gamma=torch.ones(D))


@pytest.mark.parametrize("name,bad,words", [
    ("q", _bf(T, H * D + 8), "no whole heads"), ("q", _bf(H * D, T).T, "do not lie side by side"), ("k", _bf(T - 1, HK * D), "k: fewer rows"),
    ("v", _bf(T - 1, HK * D), "v: fewer rows"), ("k", _bf(T, HK * D - D), "k: fewer rows than q, or heads"), ("v", _bf(HK * D, T).T, "side by side"),
    ("q_out", _bf(T - 1, H * D), "q_out has"), ("q_out", _bf(T, H * D + D)[:, :H * D], "q_out is not contiguous"),
    ("v_cache", _bf(PAGES - 1, PAGE, HK, D), "v_cache has"), ("k_cache", _bf(PAGES, PAGE, HK, 2 * D)[..., :D], "k_cache is not contiguous"),
    ("v_cache", _bf(PAGES, HK, PAGE, D).transpose(1, 2), "v_cache is not contiguous"), ("slots", torch.zeros(T - 1, dtype=torch.int64), "slots has"),
    ("slots", _i32(T), "slots: elements of 4"), ("positions", _i32(T - 1), "positions has 9"), ("positions", _i32(3, T - 1), "positions has 9 columns"),
    ("positions", _i32(T, 3).T, "positions: the elements of a row"), ("positions", torch.zeros(T, dtype=torch.int64), "positions: elements of 8"),
    ("positions", torch.zeros(2, T, dtype=torch.int64), "positions: elements of 4 bytes"), ("positions", _i32(T, 2)[:, 0], "positions is not contiguous"),
    ("q_gamma", torch.ones(D - 1), "q_gamma has"), ("k_gamma", _bf(D), "k_gamma: elements of 2")])
def test_qk_norm_rope(name, bad, words):
    _refused(emb.emb_qk_norm_rope, QK, name, bad, words)


ATTN = dict(Q=_bf(T, H * D), k_cache=_bf(PAGES, PAGE, HK, D), v_cache=_bf(PAGES, PAGE, HK, D), table=_i32(R, WIDTH), q_start=_i32(R + 1),
            kv_len=_i32(R), O=_bf(T, H * D), scale=0.1, max_q=4, workspace=torch.zeros(emb.EMB_PAGED_WORKSPACE, dtype=torch.uint8), prefix=_i32(R))


@pytest.mark.parametrize("name,bad,words", [
    ("Q", _bf(T, H * D + 8), "no whole heads"), ("Q", _bf(T, 2 * H * D)[:, :H * D], "Q is not contiguous"), ("O", _bf(T, 2 * H * D)[:, :H * D], "O is not contiguous"),
    ("O", _bf(T - 1, H * D), "O has"), ("O", torch.zeros(T, H * D), "O: elements of 4"), ("Q", torch.zeros(T, H * D), "Q: elements of 4"),
    ("k_cache", _bf(PAGES, HK, PAGE, D).transpose(1, 2), "k_cache is not contiguous"), ("v_cache", _bf(PAGES, PAGE, HK - 1, D), "v_cache has"),
    ("v_cache", _bf(PAGES, PAGE, HK, 2 * D)[..., :D], "v_cache is not contiguous"), ("table", _i32(R, WIDTH + 1)[:, :WIDTH], "table is not contiguous"),
    ("table", torch.zeros(R, WIDTH, dtype=torch.int64), "table: elements of 8"), ("q_start", _i32(R), "q_start has 3 elements, 4 needed"),
    ("kv_len", _i32(R - 1), "kv_len has"), ("prefix", _i32(R - 1), "prefix has"), ("kv_len", _i32(R, 2)[:, 1], "kv_len is not contiguous"),
    ("q_start", torch.zeros(R + 1, dtype=torch.int64), "q_start: elements of 8")])
def test_attention(name, bad, words):
    _refused(emb.emb_paged_attention, ATTN, name, bad, words)
