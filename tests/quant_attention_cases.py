"""Batches for each way that the attention over an 8-bit cache can take, and the
way that the library takes for a batch."""

from paper_2608_26140_amd import acache as A

# way: (what, H, Hkv, rows, keys, with a workspace)
WAYS = {
    "narrow": ("32-query kernel", 4, 2, [300], [320], True),
    "narrow split": ("32-query kernel, key splits", 4, 2, [9, 3], [1500, 700], True),
    "wide": ("256-query kernel", 4, 4, [256] * 64, [320] * 64, True),
    "wide split": ("256-query kernel, key splits", 28, 4, [256, 200], [5120, 4999], True),
    "rest 64": ("256-query tiles, up to 64 of a request left", 8, 1, [130] * 64, [300] * 64, True),
    "rest 128": ("256-query tiles, up to 128 of a request left", 32, 32, [1089, 1089], [300, 300], True),
    "rest 255": ("256-query tiles, up to 255 of a request left", 32, 32, [654] * 4, [1000] * 4, True),
}


def cu(n):
    return [int(sum(n[:i])) for i in range(len(n) + 1)]


def way_of(dims, rows, keys, ws_bytes):
    wide, narrow, rest, splits = A.acache_quant_attention_schedule(dims, cu(rows), cu(keys), ws_bytes)
    if wide and narrow:
        assert splits == 1
        return f"rest {rest}"
    return ("wide" if wide else "narrow") + (" split" if splits > 1 else "")
