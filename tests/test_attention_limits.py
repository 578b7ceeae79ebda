"""More of what attention and caches held in 4 bits refuse (no GPU is touched: every call ends before a launch)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

import paper_2504_08009_amd as oz
from test_attention_arguments import INT64, P, attention, cache, ref, rows, sequences


def test_numbers_of_tokens_whose_products_pass_64_bits():
    for tokens in (INT64, 1 << 62, 1 << 63 - 16, (1 << 26) + 1, (1 << 25) + 1):
        on = sequences(tokens=tokens)
        assert oz.lib().oz2_kv4_append(ref(cache()), ref(on), None, ref(rows(P, 128, 64)), ref(rows(P << 1, 128, 64)), None, None, None) == -2
        assert oz.lib().oz2_kv4_attention(ref(cache()), ref(on), 8, 0.1, ref(rows(P, 512, 64)), ref(rows(P << 1, 512, 64)), None) == -2
    assert attention(tokens=(1 << 25) + 1) == -4 and attention(tokens=(1 << 28) + 1) == -1
    assert attention(sequences=1 << 20, heads=16, kv_heads=16) == -2


def test_results_between_heads_that_are_not_apart():
    """heads further apart than tokens: a head of the result has to lie between two of the others"""
    # 5 tokens of 128 bf16, 256 bytes each, 1280 in all; heads 4096 bytes apart
    major = lambda at: rows(at, 128, 2048)
    far = dict(k=rows(P << 4, 256), v=rows(P << 5, 256))
    for by in (0, 256, 1278, 4096 - 1278, 4096, 7 * 4096 + 1278):
        assert attention(tokens=5, q=major(P), out=major(P + by), **far) == -12
    for by in (1278, 200 - 4096 * 3, -200):  # (one kv head, whose tokens do not lie between two heads of the result)
        assert attention(tokens=5, kv_heads=1, q=rows(P << 6), k=major(P), v=rows(P << 4, 256), out=major(P + by)) == -12
    assert attention(tokens=5, q=major(P), out=rows(P + 1280, 128, 2049), **far) == -12


def test_more_places_than_a_grid_has_chunks_of():
    c = cache(page_size=4096, codes_head=4096 * 32, codes_page=2 * 4096 * 32, scales_head=4096, scales_page=2 * 4096)
    far = dict(table=P, ld_table=1 << 20, positions=None, weights=None)
    assert oz.lib().oz2_kv4_attention(ref(c), ref(sequences(max_pages=65536, **far)), 8, 0.1, ref(rows(P, 512, 64)), ref(rows(P << 1, 512, 64)), None) == -2
    assert oz.lib().oz2_kv4_attention_workspace_bytes(ref(c), 1, 65535, 1, 2, 1) > 0 and oz.lib().oz2_kv4_attention_workspace_bytes(ref(c), 1, 65536, 1, 2, 1) == 0
    assert oz.lib().oz2_kv4_evict_workspace_bytes(ref(c), 1, 65535, 100) > 0 and oz.lib().oz2_kv4_evict_workspace_bytes(ref(c), 1, 65536, 100) == 0


def test_more_rows_over_a_cache_than_a_grid_has_workgroups_for():
    q = lambda heads: ref(rows(P, 64 * heads, 64))
    for tokens, heads, rc in ((1 << 22, 4, -3), ((1 << 22) + 1, 2, -3), (3, 1 << 22, -3)):
        assert oz.lib().oz2_kv4_attention(ref(cache()), ref(sequences(tokens=tokens)), heads, 0.1, q(heads), q(heads), None) == rc
        assert oz.lib().oz2_kv4_attention_workspace_bytes(ref(cache()), 3, 4, tokens, heads, 0) == 0
    assert oz.lib().oz2_kv4_attention_workspace_bytes(ref(cache()), 3, 4, 1 << 22, 2, 0) > 0
