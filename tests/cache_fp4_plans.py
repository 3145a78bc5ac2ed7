"""Calls of attention over a cache in 4 bits, small ones, that reach every form that it has: who shares what, how many wavefronts and tiles, one part or several.  The forms are chosen by
what the host says of a call (sequences, max_tokens, max_length), so that sequences that bring nothing, and bounds above what comes, stand in for large ones."""

KV = 2


def case(form, group, fresh, lengths, empty=0, window=0, **bounds):
    return dict(form=form, group=group, fresh=fresh + [0] * empty, lengths=(lengths + [40, 3] + [0] * empty)[:len(lengths) + empty], window=window, bounds=bounds)


CASES = []
# Up to 64 rows of a KV head, by eight wavefronts where KV heads times sequences are 32 at most, else by four; rows that fill their tiles, and that do not.
for tokens, group, tiles in ((1, 7, 1), (2, 8, 1), (3, 7, 2), (4, 8, 2), (3, 11, 3), (6, 8, 3), (7, 7, 4), (8, 8, 4), (64, 1, 4)):
    few = [tokens, 1, tokens, max(1, tokens - 1)]
    CASES += [
        case("tokens over 8 wavefronts, tiles %d, parts 1" % tiles, group, few, [500, 33, tokens, 290]),
        case("tokens over 8 wavefronts, tiles %d, parts 1" % tiles, group, few, [500, 33, tokens, 290], window=37),
        case("tokens over 8 wavefronts, tiles %d, parts 2" % tiles, group, few, [2300, 70, 1101, 1500]),
        case("tokens over 4 wavefronts, tiles %d, parts 1" % tiles, group, few, [700, 33, tokens, 290], empty=13),
        case("tokens over 4 wavefronts, tiles %d, parts 1" % tiles, group, few, [700, 33, tokens, 290], empty=13, window=200),
        case("tokens over 4 wavefronts, tiles %d, parts 2" % tiles, group, few, [1400, 70, 1101, 600], empty=13),
        case("tokens over 4 wavefronts, tiles %d, parts 2" % tiles, group, few, [1700, 70, 1101, 600], empty=13, window=1210)]
# As many parts as there are, where one of them is short; eight wavefronts.
CASES += [case("tokens over 8 wavefronts, tiles 1, parts 16", 4, [1], [17000]), case("tokens over 8 wavefronts, tiles 1, parts 64", 4, [2, 1], [9000, 3000], max_length=131072)]
# More rows: prompts by themselves, and chunks over what the cache holds, the longest sequences first up to 64 of them.
for most, alone, tiles in ((300, 260, 1), (3000, 5000, 2), (8000, 8000, 3)):
    for group in (4, 5):
        CASES += [case("rows over 4 wavefronts, tiles %d, parts 1" % tiles, group, [300, 70, 17, 1], [300, 95, 17, 1], max_tokens=most, max_length=most),
                  case("rows over 4 wavefronts, tiles %d, parts 1" % tiles, group, [260], [260], window=50 if tiles == 1 else 0, max_tokens=alone, max_length=alone)]
for group, empty, tiles, parts, most, longest in ((4, 0, 1, 21, 40, 3000), (8, 60, 1, 1, 32, 1200), (8, 17, 2, 4, 40, 4000), (8, 60, 2, 3, 40, 4000), (8, 60, 2, 1, 60, 3000), (8, 28, 3, 4, 40, 15000),
                                                  (8, 60, 3, 4, 40, 15000), (8, 60, 3, 1, 90, 15000)):
    for window in (0, longest - most) if longest < 2500 else (0,):
        CASES.append(case("rows over 4 wavefronts, tiles %d, parts %d, longest first" % (tiles, parts), group, [32, 31, 7, 1], [1700, 2500, 900, 1300], empty, window, max_tokens=most, max_length=longest))
CASES += [case("rows over 4 wavefronts, tiles 3, parts 1", 8, [40, 9], [700, 300], 90, max_tokens=60, max_length=15000),
          case("rows over 4 wavefronts, tiles 3, parts 3", 8, [40, 9], [1700, 300], 90, max_length=15000)]


def sizes(c, dim):
    from paper_2511_10909_amd import binding as mm
    return mm.BF16, dict(dict(dim=dim, heads=KV * c["group"], kv_heads=KV, page_tokens=64, pages=1000, sequences=len(c["fresh"]), table_stride=1000,
                              tokens=sum(c["fresh"]), max_tokens=max(c["fresh"]), max_length=max(c["lengths"]), window=c["window"]), **c["bounds"])
