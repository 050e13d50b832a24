"""Long calls of the attention over the paged cache, by the way their work is cut.
Sequence b reads one of two histories (b % 2), of which it holds its first lens[b] keys.

name: (types, D, H, Hkv, causal, page, lens, news, what the call's plan must reach)
types: the caches ("bf", "mx") for which the plan is that one.  news None: one token each.
The last entry, over the fields of tests/paged_plan_host.cpp's output: rows, host_whole,
whole, units, run, piece (key blocks), most (units of a workgroup), cut, blocks."""

# 1 to 4 tokens for most, a few prompts; 100 sequences
_RAGGED = [(37 * b * b) % 9000 + 1 for b in range(100)]

CASES = {
    # units kept whole by the workgroups' own sums, two or more each, early and late tiles in turn
    "whole_few": (("bf", "mx"), 64, 16, 4, True, 16, [1100 + b % 100 for b in range(384)], None,
                  lambda p: p.rows == 16 and not p.host_whole and p.whole and p.most >= 3),
    "whole_few_long": (("bf", "mx"), 64, 8, 4, True, 64, [16700 - b for b in range(256)], None,
                       lambda p: p.whole and p.piece > 2 * 256),        # page numbers asked for three times
    "whole_rows": (("bf",), 64, 4, 4, True, 32, [2000 + b for b in range(192)], [33 + b % 5 for b in range(192)],
                   lambda p: p.rows == 256 and not p.host_whole and p.whole and p.most >= 3),
    "whole_rows_mx": (("mx",), 64, 8, 4, True, 32, [2200 - b for b in range(192)], [65 + b % 5 for b in range(192)],
                      lambda p: p.rows == 256 and p.whole and p.most >= 3 and p.piece > 32),
    "whole_rows_long": (("bf",), 128, 4, 4, True, 16, [9000 - 3 * b for b in range(64)], [34] * 64,
                        lambda p: p.rows == 256 and p.whole and p.piece > 2 * 64),
    "whole_prompts": (("bf", "mx"), 64, 4, 2, True, 64, [1500] * 40, [1500 - 9 * b for b in range(40)],
                      lambda p: p.rows == 256 and not p.host_whole and p.whole and p.most >= 3),
    # a line that is cut, of more sequences than lanes
    "cut_few": (("bf", "mx"), 128, 8, 2, True, 16, _RAGGED, None,
                lambda p: p.rows == 16 and not p.whole and p.cut > 60 and p.run > 8),
    "cut_few_drafts": (("bf", "mx"), 64, 8, 2, True, 16, _RAGGED, [1 + b % 9 for b in range(100)],
                       lambda p: p.rows == 32 and not p.whole and p.cut > 60),
    "cut_mx_64": (("mx",), 64, 8, 2, True, 16, _RAGGED, [8 + b % 9 for b in range(100)],
                  lambda p: p.rows == 64 and not p.whole and p.cut > 60),
    "cut_rows": (("bf",), 64, 8, 2, True, 16, _RAGGED, [9 + b % 30 for b in range(100)],
                 lambda p: p.rows == 256 and not p.whole and p.cut > 60 and p.run > 4),
    "cut_rows_mx": (("mx",), 64, 8, 2, True, 16, _RAGGED, [30 + b % 30 for b in range(100)],
                    lambda p: p.rows == 256 and not p.whole and p.cut > 60 and p.run > 4),
    # long runs: page numbers are asked for again inside a piece
    "long_few": (("bf", "mx"), 64, 4, 4, True, 1024, [600000, 590001, 1], [1, 1, 1],
                 lambda p: p.rows == 16 and not p.whole and p.run > 256 and p.piece > 256),
    "long_mx_64": (("mx",), 64, 4, 4, False, 1024, [300000, 280001], [40, 33],
                   lambda p: p.rows == 64 and not p.whole and p.piece > 128),
    "long_rows": (("bf",), 64, 4, 4, True, 128, [140000, 133333], [50, 41],
                  lambda p: p.rows == 256 and not p.whole and p.piece > 64),
    "long_rows_mx": (("mx",), 128, 2, 2, True, 128, [100000, 80001], [300, 270],
                     lambda p: p.rows == 256 and not p.whole and p.piece > 32),
}
