"""What reads the prefixes of a shared_attention call, by its sizes: the rule of way_of in kf_shared_attention.cu (held to it by
test_shared_ways_host.py), and cases whose sizes choose each way."""

MB = 1 << 20


def way_of(B, rows, Hq, Hkv, hd, n_pages, page, width, n):
    per = rows * (Hq // Hkv)
    tiles = 2 * (B * -(-per // 16) + n + 1) * Hkv
    counted = n <= 1 << 24 and B * rows * Hq <= 1 << 30 and tiles <= 1 << 30 and tiles * (width * page // 16 + 8) <= 0x7fffffff
    if n >= B or n_pages == 0 or not counted:
        return "paged"
    seg = 32 if hd == 64 and per > 16 else 16
    keys = min(width, n_pages) * page * hd * 4 * Hkv
    if B * -(-per // seg) * keys <= 48 * MB:
        return "paged"
    return "rows" if ((B * per + seg - 1) // seg + n) * keys <= 128 * MB else "tiles"


# (groups of (prefix, lengths), rows, query heads, KV heads, head_dim), and how many pages more the table and the pool have
def _many(n, rows, at=700, more=10):
    return [(at, [at + more + i for i in range(n)]), (64, [72] * 9)], rows, 24, 4, 64


def _spread(n):
    return [(17 * i, [17 * i + 1 + j for j in range(1 + i % 4)]) for i in range(n)], 1, 3, 3


CASES = {
    "paged": [
        (*([(1000, [1000 + i for i in range(11)])], 1, 32, 8), 64, 0), (*([(1000, [1000 + i for i in range(11)])], 1, 32, 8), 128, 0),
        ([(4000, [4010 + 9 * i for i in range(4)])], 3, 16, 2, 64, 0), ([(4000, [4010 + 9 * i for i in range(4)])], 3, 16, 2, 128, 0),
        (*_spread(20), 64, 0), (*_spread(20), 128, 0), ([(63, [64 + i for i in range(60)])], 2, 8, 4, 128, 0),
        ([(8000, [8001 + 30 * i for i in range(4)])], 1, 8, 2, 128, 0), (*_many(20, 8), 0),
        ([(333, [340, 900, 341]), (48, [56, 57]), (5, [13, 14, 15, 40])], 8, 8, 2, 128, 0),
    ],
    "rows": [
        # many sequences a group, several tiles of rows, tiles of 32 (head_dim 64, more than 16 rows a sequence)
        (*_many(80, 8), 0), ([(517, [518 + 7 * i for i in range(100)])], 1, 12, 4, 64, 0), ([(300, [300 + i for i in range(200)])], 1, 16, 2, 64, 0),
        ([(4000, [4010 + 9 * i for i in range(40)])], 3, 16, 2, 64, 0), ([(4000, [4010 + 9 * i for i in range(16)])], 3, 16, 2, 128, 0),
        # a prefix in more pieces than warps take whole
        ([(32771, [32772 + 100 * i for i in range(6)])], 1, 8, 2, 128, 0), ([(20011, [20012 + 100 * i for i in range(9)]), (1, [3, 2])], 1, 8, 2, 64, 0),
        # many groups of few sequences, prefixes of none to 663 tokens; groups of none
        (*_spread(40), 64, 40), (*_spread(30), 128, 8), ([(0, []), (250, [260] * 30), (9, []), (31, [40] * 40), (4, [])], 4, 12, 3, 64, 60),
        # a table far wider than the sequences
        ([(16, [17, 40, 31])], 1, 8, 8, 64, 600), ([(129, [131, 300]), (5, [6])], 5, 8, 2, 128, 1200),
    ],
    "tiles": [
        (*_many(150, 8), 0), ([(32771, [32772 + 100 * i for i in range(6)])], 1, 8, 2, 128, 2100),
        ([(4000, [4010 + 9 * i for i in range(40)])], 3, 16, 2, 128, 0), ([(1000, [1000 + i for i in range(64)])], 1, 32, 8, 128, 200),
        (*_spread(40), 128, 100), ([(0, []), (250, [260] * 30), (9, []), (31, [40] * 40), (4, [])], 4, 12, 3, 128, 200),
        ([(16, [17, 40, 31])], 1, 8, 8, 64, 2100),
        # one sub-tile alone, a pair and a row, rows of many groups in one CTA
        ([(700, [701 + i for i in range(127)])], 1, 4, 4, 64, 900), ([(700, [701 + i for i in range(257)])], 1, 4, 4, 128, 400),
        ([(200 + i, [210 + i, 300]) for i in range(60)], 2, 8, 4, 64, 300),
    ],
}


def sizes_of(case, page=16):
    """The arguments of way_of for a case, as test_gpu_shared_attention.make lays it out with two columns and three pages to spare."""
    groups, rows, Hq, Hkv, hd, more = case
    pages = sum(n // page + sum(-(-x // page) - n // page for x in lens) for n, lens in groups) + 3 + more
    width = max(-(-x // page) for _, lens in groups for x in lens) + 2 + more
    return sum(len(lens) for _, lens in groups), rows, Hq, Hkv, hd, pages, page, width, len(groups)
