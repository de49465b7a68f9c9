"""Sizes that take attention of many rows through each of its kernels, on 256 compute units."""
import paper_2511_04214_amd as brq

# sequences, heads of the cache, max_kv; "tall" has more tiles of 128 rows than units, but not more tiles of 256
FORMS = {"one": (12, 2, 384), "pair": (12, 2, 500), "pair in parts": (12, 2, 1000), "tall": (12, 18, 500)}
GROUPED = dict(FORMS, tall=(12, 14, 500))                    # of 3 query heads to each
# besides: rows of each sequence
NAN = {"one": (12, 2, 384, 40), "pair": (12, 2, 500, 40), "pair in parts": (12, 2, 1000, 40), "tall": (4, 32, 500, 300)}


def plan(form, D, forms, T, max_q, causal=True, window=0, G=1, cus=256):
    S, Hk, max_kv = forms[form]
    return brq.diag_kv4_attention_route(T, S, G * Hk, Hk, D, max_q, max_kv, causal, window, cus)
