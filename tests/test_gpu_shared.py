"""specvlm_pages_shared, specvlm_shared_attn and specvlm_cross_attn against plain implementations in 64 bits."""
import numpy as np
import pytest
import torch

import shared_reference as S
from gpu_util import dev_bf16, host_f64, rnd_bits

pytestmark = pytest.mark.gpu
POISON = 0x7fc1                                     # a bf16 NaN: what rows that nobody wrote may hold


@pytest.fixture(scope="module")
def B():
    from paper_2508_16201_amd import binding
    binding.lib()
    return binding


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def build(seed, videos, heads, ps, spare=3):
    """videos: [(tokens of whole pages that are shared, [(own tokens, block) of each request])].  Pages in no order; rows and pages that belong to no
    token are poisoned -> (q, k, v, table, kv_lens, q_lens, groups)."""
    hq, hkv, d = heads
    rng = np.random.default_rng(seed)
    requests = [(shared, own, ql, len(video)) for shared, video in videos for own, ql in video]
    kv_lens, q_lens = [shared + own for shared, own, _, _ in requests], [ql for _, _, ql, _ in requests]
    total = sum(shared // ps + sum(-(-own // ps) for own, _ in video) for shared, video in videos) + spare
    ids, at = rng.permutation(total).astype(np.int32), 0
    width = max(-(-n // ps) for n in kv_lens)
    table = np.full((len(requests), width), -1, dtype=np.int32)
    k = np.full((total, ps, hkv, d), POISON, dtype=np.uint16)
    v = k.copy()
    groups, b = np.zeros((3, len(requests)), dtype=np.int32), 0

    def fill(pages, tokens, salt):
        for i, page in enumerate(pages):
            rows = min(ps, tokens - i * ps)
            k[page, :rows] = rnd_bits((rows, hkv, d), (seed, salt, i, 1))
            v[page, :rows] = rnd_bits((rows, hkv, d), (seed, salt, i, 2))

    for shared, video in videos:
        common, at = ids[at:at + shared // ps], at + shared // ps
        fill(common, shared, 1000 + b)
        first = b
        for own, _ in video:
            mine, at = ids[at:at + -(-own // ps)], at + -(-own // ps)
            fill(mine, own, b)
            table[b, :len(common) + len(mine)] = np.concatenate([common, mine])
            alone = len(video) == 1 or shared == 0
            groups[:, b] = (b, 1, 0) if alone else (first, len(video) if b == first else 0, shared)
            b += 1
    return rnd_bits((sum(q_lens), hq, d), (seed, 3)), k, v, table, kv_lens, q_lens, groups


def pool(x, head_major):
    return dev_bf16(np.ascontiguousarray(x.transpose(0, 2, 1, 3))).transpose(1, 2) if head_major else dev_bf16(x)


def ragged(q_lens, **more):
    return dict(cu_q=i32(np.concatenate([[0], np.cumsum(q_lens)])), max_q_len=max(q_lens), **more)


def close(got, want, tol, written=None):
    written = np.ones(len(got), dtype=bool) if written is None else written
    err = np.abs(got - want)[written]
    assert np.isfinite(got[written]).all()
    assert (err <= tol[written]).all(), (err - tol[written]).max()


def check(B, q, k, v, table, kv_lens, q_lens, groups, *, head_major=False, masks=None, parts=1, scale=None, **kw):
    scale = q.shape[2] ** -0.5 if scale is None else scale
    want, want_lse, tol, tol_lse, written = S.shared_attention(S.values(q), S.values(k), S.values(v), table, kv_lens, q_lens, scale, masks, parts,
                                                               kw.get("max_kv_len"), kw.get("max_q_len"))
    more = dict(kw)
    if len(set(q_lens)) > 1 and "cu_q" not in kw:
        more.update(ragged(q_lens))
    if masks is not None:
        more["ancestor_mask"] = torch.from_numpy(np.asarray(masks, dtype=np.uint64).view(np.int64)).cuda()
    qd = dev_bf16(q)
    out = torch.full_like(qd, 7.0)
    got, lse = B.shared_attn(qd, pool(k, head_major), pool(v, head_major), i32(table), i32(kv_lens), scale, i32(groups), out=out, want_lse=True, **more)
    torch.cuda.synchronize()
    assert got is out
    got, lse = host_f64(got), host_f64(lse)
    assert (got[~written] == 7.0).all()
    close(got, want, tol, written)
    none = np.isinf(want_lse) & written[:, None]
    assert (lse[none] == -np.inf).all() and (got[none] == 0).all()
    some = ~none & written[:, None]
    assert (np.abs(lse[some] - want_lse[some]) <= tol_lse[some]).all()
    return got


HEADS = [(4, 1, 64), (14, 2, 64), (3, 3, 64), (28, 4, 128), (16, 2, 128), (5, 5, 128)]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("shared,ps,own,block", [(16, 16, 1, 1), (32, 32, 5, 2), (48, 48, 40, 1), (128, 64, 130, 6), (144, 16, 17, 17), (320, 16, 200, 33),
                                                 (256, 256, 31, 5)])
def test_a_group(B, heads, shared, ps, own, block):
    args = build(shared + own, [(shared, [(own + i, block) for i in range(3)])], heads, ps)
    check(B, *args)
    check(B, *args, head_major=True)


@pytest.mark.parametrize("heads", [(14, 2, 64), (28, 4, 128)])
def test_groups_and_requests_alone_of_all_lengths(B, heads):
    """Two to four requests about a video, blocks of different lengths, requests alone between them, one token and long ones."""
    args = build(7, [(160, [(9, 3), (30, 1)]), (0, [(1, 1)]), (0, [(150, 2)]), (304, [(5, 5), (80, 40), (16, 1), (17, 2)]), (0, [(16, 16)]), (16, [(2, 2), (1, 1)])],
                 heads, 16)
    check(B, *args)


@pytest.mark.parametrize("members,heads,block", [(2, (64, 8, 128), 1), (4, (64, 8, 128), 1), (3, (8, 1, 64), 9), (9, (64, 8, 128), 4), (17, (4, 1, 64), 7), (33, (16, 2, 64), 1)])
def test_rows_of_a_set(B, members, heads, block):
    """16 to 480 rows of a kv head meet the shared keys: one to eight waves' worth of them, and more than a set."""
    args = build(members, [(496, [(block + 3 * i, block) for i in range(members)])], heads, 16)
    check(B, *args)


def test_few_rows_keep_probabilities_in_two_parts(B):
    args = build(5, [(1600, [(60, 2), (70, 2)])], (14, 2, 64), 16)
    check(B, *args, parts=2)


@pytest.mark.parametrize("heads,shared,members", [((28, 4, 128), 6000, 3), ((14, 2, 64), 9008, 5), ((16, 2, 128), 4096, 20)])
def test_long_keys_are_cut_and_joined(B, heads, shared, members):
    args = build(shared, [(shared, [(20 + 40 * i, 1 + i % 3) for i in range(members)])], heads, 16)
    check(B, *args)


@pytest.mark.parametrize("q_len", [63, 64, 65, 200, 517])
def test_whole_questions(B, q_len):
    """Blocks longer than a mask has bits, and than a set has rows."""
    args = build(q_len, [(336, [(q_len, q_len), (q_len + 30, q_len // 2)]), (0, [(q_len, q_len)])], (4, 1, 64), 48)
    check(B, *args)


@pytest.mark.parametrize("heads", [(4, 1, 64), (28, 4, 128)])
@pytest.mark.parametrize("nodes", [1, 9, 26, 64])
def test_trees(B, heads, nodes):
    from paper_2508_16201_amd import synth
    masks = np.concatenate([np.asarray(synth.ancestor_masks(synth.make_tree(nodes, 3 + i))).astype(np.uint64) for i in range(3)])
    args = build(nodes, [(96, [(nodes, nodes), (nodes + 45, nodes), (nodes + 16, nodes)])], heads, 16)
    check(B, *args, masks=masks)


def test_a_node_that_sees_nothing_of_its_block(B):
    args = build(3, [(16, [(3, 3), (4, 3)]), (0, [(3, 3)])], (4, 1, 64), 16)
    check(B, *args, masks=np.array([0, 3, 5, 1, 2, 0, 0, 0, 7], dtype=np.uint64))


def test_more_requests_than_a_workgroup_has_threads(B):
    """600 requests in 200 groups: 1200 entries."""
    args = build(11, [(32, [(1 + (i + j) % 20, 1) for j in range(3)]) for i in range(200)], (2, 1, 64), 16)
    check(B, *args)


@pytest.mark.parametrize("batch", [255, 256, 257])
def test_as_many_requests_as_threads(B, batch):
    args = build(batch, [(16, [(1 + i % 3, 1) for i in range(batch - 1)]), (0, [(9, 1)])], (2, 1, 64), 16)
    check(B, *args)


def test_rows_that_are_left_alone(B):
    """Requests with no block, with a longer one than their cache, with more tokens than the call says, rows behind the last request."""
    q, k, v, table, kv_lens, q_lens, groups = build(5, [(64, [(10, 2), (12, 3), (4, 2)]), (0, [(40, 3)]), (0, [(50, 4)])], (4, 2, 64), 16)
    q = np.concatenate([q, q[:5]])
    kv_lens = [74, 76, 1, 90, 50]                           # the third is shorter than what it shares, the fourth longer than the call allows
    more = dict(cu_q=i32([0, 2, 5, 7, 10, 14]), max_q_len=4, max_kv_len=80)
    scale = 0.125
    want, want_lse, tol, _, written = S.shared_attention(S.values(q)[:14], S.values(k), S.values(v), table, kv_lens, q_lens, scale, max_kv=80, max_q=4)
    assert written.sum() == 9
    out = torch.full((19, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    B.shared_attn(dev_bf16(q), dev_bf16(k), dev_bf16(v), i32(table), i32(kv_lens), scale, i32(groups), out=out, **more)
    got = host_f64(out)
    assert (got[14:] == 7.0).all() and (got[:14][~written] == 7.0).all()
    close(got[:14], want, tol, written)


NOT_GROUPS = {"beyond the batch": (0, 9, 64), "more than lies before a block": (0, 3, 96), "no multiple of 16": (0, 3, 40), "nothing": (0, 3, 0), "negative": (0, 3, -64),
              "one": (0, 1, 64), "of another first": (1, 3, 64), "far": (1 << 30, 1 << 30, 1 << 30), "below": (-5, -5, -5)}


@pytest.mark.parametrize("what", NOT_GROUPS)
def test_what_is_no_group_is_left_out(B, what):
    q, k, v, table, kv_lens, q_lens, groups = build(6, [(64, [(10, 2), (12, 3), (30, 2)])], (4, 2, 64), 16)
    first, members, shared = NOT_GROUPS[what]
    groups[0], groups[1, 0], groups[2] = first, members, shared
    check(B, q, k, v, table, kv_lens, q_lens, groups)


def test_groups_that_overlap_are_left_out(B):
    """Every request the first of a group of all behind it: their rows would be there many times."""
    q, k, v, table, kv_lens, q_lens, groups = build(6, [(64, [(10, 9)] * 40)], (4, 1, 64), 16)
    groups[0] = np.arange(40)
    groups[1] = 40 - np.arange(40)
    check(B, q, k, v, table, kv_lens, q_lens, groups)


def test_a_member_with_a_shorter_cache_is_taken_alone(B):
    """Its block begins inside what the others share."""
    q, k, v, table, kv_lens, q_lens, groups = build(8, [(128, [(10, 2), (12, 3), (30, 2)])], (4, 2, 64), 16)
    kv_lens[1] = 100
    check(B, q, k, v, table, kv_lens, q_lens, groups)


@pytest.mark.parametrize("heads", [(4, 1, 64), (16, 2, 128)])
@pytest.mark.parametrize("odd", [-1, 999, -2147483648])
def test_pages_that_are_none(B, heads, odd):
    """Of the shared ones and of a request's own; all of a request's but its block's."""
    q, k, v, table, kv_lens, q_lens, groups = build(9, [(320, [(40, 2), (12, 3), (30, 2)]), (0, [(40, 1)])], heads, 16)
    table[:3, [0, 3, 7, 8, 9]] = odd
    table[0, 20] = odd
    table[3, :2] = odd
    check(B, q, k, v, table, kv_lens, q_lens, groups)
    table[:3, :20] = odd
    table[3, 2] = odd                                       # nothing left
    check(B, q, k, v, table, kv_lens, q_lens, groups)


def test_the_other_rows_of_a_group_name_no_pages_there(B):
    """The shared pages are those of the group's first request."""
    args = build(10, [(160, [(9, 3), (30, 1), (4, 4)])], (14, 2, 64), 16)
    q, k, v, table, kv_lens, q_lens, groups = args
    want = check(B, *args)
    table = table.copy()
    table[1:, :10] = -1
    got = B.shared_attn(dev_bf16(q), dev_bf16(k), dev_bf16(v), i32(table), i32(kv_lens), 0.125, i32(groups), **ragged(q_lens))
    assert (host_f64(got) == want).all()


def bits(x):
    from paper_2508_16201_amd.synth import f32_to_bf16_bits
    return f32_to_bf16_bits(np.asarray(x, dtype=np.float32))


@pytest.mark.parametrize("heads,members", [((4, 1, 64), 2), ((16, 2, 128), 2), ((16, 2, 128), 40)])
@pytest.mark.parametrize("place", [0, 100, 319, 322])
def test_values_that_are_no_finite_numbers(B, heads, members, place):
    """What a row sees of them comes out, however small its weight; place 322 is a request's own key."""
    q, k, v, table, kv_lens, q_lens, groups = build(12, [(320, [(20, 2)] * members)], heads, 16)
    k[table[0, place // 16], place % 16] = bits(-5.0 * np.sign(S.values(q[0, 0]) + 1e-3))      # (a weight of the first row that 32 bits take for 0)
    flat = v.copy()
    v[table[0, place // 16], place % 16, :, 3], v[table[0, place // 16], place % 16, :, 9] = 0x7f80, 0xff80
    v[table[0, place // 16], place % 16, :, 20] = 0x7fc0
    flat[table[0, place // 16], place % 16][:, [3, 9, 20]] = 0
    want, _, tol, _, _ = S.shared_attention(S.values(q), S.values(k), S.values(flat), table, kv_lens, q_lens, 0.5)
    got = host_f64(B.shared_attn(dev_bf16(q), dev_bf16(k), dev_bf16(v), i32(table), i32(kv_lens), 0.5, i32(groups)))
    rows = np.arange(len(q)) < (len(q) if place < 320 else 2)
    plain = [c for c in range(heads[2]) if c not in (3, 9, 20)]
    assert (np.abs(got - want)[:, :, plain] <= tol[:, :, plain]).all()
    assert (got[rows][:, :, 3] == np.inf).all() and (got[rows][:, :, 9] == -np.inf).all() and np.isnan(got[rows][:, :, 20]).all()
    assert (np.abs(got - want)[~rows] <= tol[~rows]).all()


@pytest.mark.parametrize("heads", [(4, 1, 64), (16, 2, 128)])
def test_hidden_values_change_nothing(B, heads):
    """Of keys behind a query in its block, of pages that are none (the pool's first is read in their place) and behind the last token."""
    q, k, v, table, kv_lens, q_lens, groups = build(13, [(320, [(20, 5), (40, 5)])], heads, 16)
    table[:, 4] = -1
    check(B, q, k, v, table, kv_lens, q_lens, groups)
    want_exact, _, tol, _, _ = S.shared_attention(S.values(q), S.values(k), S.values(v), table, kv_lens, q_lens, heads[2] ** -0.5)
    for odd in (0x7f80, 0xff80, 0x7fc0):
        k2, v2 = k.copy(), v.copy()
        for x in (k2, v2):
            x[np.setdiff1d(np.arange(len(k)), table)] = odd
            for b in range(2):
                n = kv_lens[b]
                x[table[b, (n - 1) // 16], (n - 1) % 16 + 1:] = odd
                x[table[b, (n - 1) // 16], (n - 1) % 16] = odd           # the last key: only the last query sees it
        got = host_f64(B.shared_attn(dev_bf16(q), dev_bf16(k2), dev_bf16(v2), i32(table), i32(kv_lens), heads[2] ** -0.5, i32(groups)))
        keep = [t for t in range(10) if t % 5 != 4]
        # (rows that share a product with such a value are summed once more, with probabilities in 32 bits: within the same bounds, of which those of the first
        # sum are the larger)
        close(got[keep], want_exact[keep], tol[keep])


def test_the_queries_may_be_the_output_and_strides_are_anything(B):
    q, k, v, table, kv_lens, q_lens, groups = build(14, [(96, [(20, 2), (40, 2), (9, 2)])], (6, 2, 64), 16)
    want = check(B, q, k, v, table, kv_lens, q_lens, groups)
    wide = torch.zeros((9, 6, 80), dtype=torch.bfloat16, device="cuda")[1:7, :, 8:72]
    wide.copy_(dev_bf16(q))
    big = torch.zeros((len(k), 16, 3, 64), dtype=torch.bfloat16, device="cuda")
    kd, vd = big.clone()[:, :, 1:], big[:, :, 1:]
    kd.copy_(dev_bf16(k))
    vd.copy_(dev_bf16(v))
    rows = torch.full((3, table.shape[1] + 5), -7, dtype=torch.int32, device="cuda")[:, 2:2 + table.shape[1]]
    rows.copy_(i32(table))
    B.shared_attn(wide, kd, vd, rows, i32(kv_lens), 0.125, i32(groups), out=wide)
    assert (host_f64(wide) == want).all()


def test_a_request_taken_alone_among_a_group_where_the_queries_are_the_output(B):
    """The group's pieces read its queries as long as they run: nothing is written over them before."""
    q, k, v, table, kv_lens, q_lens, groups = build(79, [(3200, [(20, 4), (17, 4), (60, 4), (33, 4)])], (28, 4, 128), 16)
    kv_lens[1] = 50                                      # (shorter than what the group shares)
    args = dev_bf16(k), dev_bf16(v), i32(table), i32(kv_lens), 0.1, i32(groups)
    want = B.shared_attn(dev_bf16(q), *args)
    exact, _, tol, _, _ = S.shared_attention(S.values(q), S.values(k), S.values(v), table, kv_lens, q_lens, 0.1)
    close(host_f64(want), exact, tol)
    first = None
    for _ in range(5):
        out = dev_bf16(q)
        B.shared_attn(out, *args, out=out)
        close(host_f64(out), exact, tol)
        first = out if first is None else first
        assert (out == first).all() and (out == want).all()


def test_a_zero_scale_takes_the_mean(B):
    args = build(15, [(96, [(20, 2), (40, 2)])], (6, 2, 64), 16)
    check(B, *args, scale=0.0)


# ------------------------------------------------------------------------------------------------ cross attention
def check_cross(B, seed, heads, q_lens, kv_lens, *, head_major=False, ranges=None, parts=1, cu=True, scale=None):
    hq, hkv, d = heads
    scale = d ** -0.5 if scale is None else scale
    q, k, v = rnd_bits((sum(q_lens), hq, d), (seed, 1)), rnd_bits((sum(kv_lens), hkv, d), (seed, 2)), rnd_bits((sum(kv_lens), hkv, d), (seed, 3))
    want, want_lse, tol, tol_lse = S.cross_attention(S.values(q), S.values(k), S.values(v), q_lens, kv_lens, scale, ranges, parts)
    side = (lambda x: dev_bf16(np.ascontiguousarray(x.transpose(1, 0, 2))).transpose(0, 1)) if head_major else dev_bf16
    more = dict(cu_q=i32(np.concatenate([[0], np.cumsum(q_lens)])), cu_kv=i32(np.concatenate([[0], np.cumsum(kv_lens)]))) if cu else {}
    if ranges is not None:
        more["key_ranges"] = i32(ranges)
    got, lse = B.cross_attn(dev_bf16(q), side(k), side(v), scale, want_lse=True, **more)
    got, lse = host_f64(got), host_f64(lse)
    close(got, want, tol)
    none = np.isinf(want_lse)
    assert (lse[none] == -np.inf).all() and (got[none] == 0).all()
    assert (np.abs(lse[~none] - want_lse[~none]) <= tol_lse[~none]).all()


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("queries,states", [(1, 1), (1, 16), (2, 31), (1, 33), (7, 127), (40, 128), (33, 129), (100, 300), (1, 1254)])
def test_one_encoder(B, heads, queries, states):
    check_cross(B, states, heads, [queries], [states], cu=False)
    check_cross(B, states, heads, [queries], [states], head_major=True)


@pytest.mark.parametrize("heads,queries,states", [((28, 4, 128), 1, 9000), ((14, 2, 64), 3, 5003), ((64, 8, 128), 70, 2100)])
def test_many_states_are_cut_and_joined(B, heads, queries, states):
    check_cross(B, states, heads, [queries], [states], cu=False)


def test_few_queries_keep_probabilities_in_two_parts(B):
    check_cross(B, 1, (28, 4, 128), [3], [2000], parts=2)


@pytest.mark.parametrize("heads", [(4, 1, 64), (28, 4, 128)])
def test_entries_of_all_lengths(B, heads):
    """None of one or the other among them: the queries of no states get nothing."""
    check_cross(B, 5, heads, [1, 0, 5, 130, 3, 0, 2], [300, 77, 1, 1000, 0, 0, 17])


def test_many_entries(B):
    n = 700
    check_cross(B, 6, (2, 1, 64), [(i * 7) % 4 for i in range(n)], [(i * 13) % 50 for i in range(n)])


@pytest.mark.parametrize("heads", [(4, 1, 64), (16, 2, 128)])
@pytest.mark.parametrize("states", [40, 1000])
def test_ranges(B, heads, states):
    """Any, empty, turned round, far outside of the entry."""
    rng = np.random.default_rng(states)
    n = [90, 150]
    ranges = np.sort(rng.integers(-20, states + 40, (sum(n), 2)), axis=1).astype(np.int32)
    ranges[::7] = [[5, 5]]
    ranges[3::11] = [[9, 4]]
    ranges[4::13] = [[-(2 ** 31), 2 ** 31 - 1]]
    ranges[5::17] = [[2 ** 31 - 1, 2 ** 31 - 1]]
    ranges[6::19] = [[states - 1, states]]
    ranges[8::23] = [[-(2 ** 31), -(2 ** 31)]]
    check_cross(B, states, heads, n, [states, states // 2], ranges=ranges)


def test_no_query_sees_anything(B):
    check_cross(B, 8, (4, 1, 64), [40], [500], ranges=np.zeros((40, 2), dtype=np.int32))


@pytest.mark.parametrize("cu", [False, True])
@pytest.mark.parametrize("ranges", [False, True])
def test_no_states_at_all(B, cu, ranges):
    q, none = dev_bf16(rnd_bits((43, 4, 64), 8)), torch.empty((0, 1, 64), dtype=torch.bfloat16, device="cuda")
    more = dict(cu_q=i32([0, 3, 43]), cu_kv=i32([0, 0, 0])) if cu else {}
    if ranges:
        more["key_ranges"] = i32(np.full((43, 2), [0, 9]))
    got, lse = B.cross_attn(q, none, none, 0.125, want_lse=True, **more)
    assert (got == 0).all() and (lse == -np.inf).all()


def test_text_between_frames(B):
    ranges = np.array([[max(0, (t // 10 - 3) * 49), t // 10 * 49] for t in range(300)], dtype=np.int32)
    check_cross(B, 9, (16, 2, 128), [300], [30 * 49], ranges=ranges)


def test_entries_that_leave_the_tensors_are_left_alone(B):
    q, k, v = dev_bf16(rnd_bits((12, 4, 64), 1)), dev_bf16(rnd_bits((100, 1, 64), 2)), dev_bf16(rnd_bits((100, 1, 64), 3))
    want = B.cross_attn(q[3:5], k[10:60], v[10:60], 0.125)
    for cu_q, cu_kv, left in (([0, 3, 5, 9], [-5, 10, 60, 101], True), ([0, 3, 5, 13], [0, 10, 60, 100], False), ([-1, 3, 5, 4], [0, 10, 60, 70], False),
                              ([0, 3, 5, 9], [20, 10, 60, 30], True)):
        out = torch.full_like(q, 7.0)
        B.cross_attn(q, k, v, 0.125, cu_q=i32(cu_q), cu_kv=i32(cu_kv), out=out)
        assert (out[3:5] == want).all() and (out[9:] == 7.0).all()
        assert not left or (out[:3] == 7.0).all() and (out[5:9] == 7.0).all()


def test_offsets_that_overlap_write_nothing(B):
    """Entries with the same queries, so many that there is no room for their results."""
    q, k = dev_bf16(rnd_bits((40, 4, 64), 1)), dev_bf16(rnd_bits((100, 1, 64), 2))
    out = torch.full_like(q, 7.0)
    cu_q = [0, 40] * 60 + [0]
    B.cross_attn(q, k, k, 0.125, cu_q=i32(cu_q), cu_kv=i32([0, 100] * 60 + [0]), out=out)
    assert (out == 7.0).all()


@pytest.mark.parametrize("paged", [False, True])
def test_offsets_that_overlap_by_more_than_an_int_holds(B, paged):
    """2^31 rows, counted with the repeated ones: as a sum of ints none."""
    batch, queries = 16384, 4096
    q, k = dev_bf16(rnd_bits((queries, 64, 64), 1)), dev_bf16(rnd_bits((4096, 1, 64), 2))
    out = torch.full_like(q, 7.0)
    cu = torch.zeros(batch + 1, dtype=torch.int32, device="cuda")
    cu[1::2] = queries
    if paged:
        table = torch.arange(256, dtype=torch.int32, device="cuda").expand(batch, 256)
        B.shared_attn(q, k.view(256, 16, 1, 64), k.view(256, 16, 1, 64), table, torch.full((batch,), 4096, dtype=torch.int32, device="cuda"), 0.125,
                      torch.zeros((3, batch), dtype=torch.int32, device="cuda"), cu_q=cu, max_q_len=queries, max_kv_len=4096, out=out)
    else:
        B.cross_attn(q, k[:64], k[:64], 0.125, cu_q=cu, cu_kv=torch.clamp(cu, max=64), out=out)
    assert (out == 7.0).all()


@pytest.mark.parametrize("queries", [2, 60])
def test_odd_values_of_states(B, queries):
    heads = (16, 2, 128)
    q, k, v = rnd_bits((queries, 16, 128), 1), rnd_bits((700, 2, 128), 2), rnd_bits((700, 2, 128), 3)
    flat = v.copy()
    v[333, :, 5], v[333, :, 6], v[40, 1, 7] = 0x7f80, 0xff80, 0x7fc0
    flat[333][:, [5, 6]], flat[40, 1, 7] = 0, 0
    ranges = np.array([[0, 700] if t % 2 else [334, 700] for t in range(queries)], dtype=np.int32)
    want, _, tol, _ = S.cross_attention(S.values(q), S.values(k), S.values(flat), [queries], [700], 0.1, ranges)
    got = host_f64(B.cross_attn(dev_bf16(q), dev_bf16(k), dev_bf16(v), 0.1, key_ranges=i32(ranges)))
    sees = np.arange(queries) % 2 == 1
    assert (got[sees][:, :, 5] == np.inf).all() and (got[sees][:, :, 6] == -np.inf).all() and np.isnan(got[sees][:, 8:, 7]).all()
    assert np.abs(got - want)[~sees].max() <= tol[~sees].max() and (np.abs(got - want)[~sees] <= tol[~sees]).all()
    plain = [c for c in range(128) if c not in (5, 6, 7)]
    assert (np.abs(got - want)[:, :, plain] <= tol[:, :, plain]).all()


def grown(k, by):
    """The keys from 300 on `by` times as long: their logits rise far above what the first tiles leave as the maximum."""
    x = S.values(k)
    x[300:] *= by
    return bits(x)


@pytest.mark.parametrize("heads", [(4, 1, 64), (16, 2, 128)])
@pytest.mark.parametrize("queries", [1, 7, 15, 30, 70])
@pytest.mark.parametrize("by", [1.0, 4.0])
def test_steep_logits(B, heads, queries, by):
    """Logits of up to a few hundred, of waves that have rows for themselves, share them by two and by four."""
    hq, hkv, d = heads
    scale = 6.0 * 8.0 / d / by
    q, k, v = rnd_bits((queries, hq, d), (51, queries)), rnd_bits((2000, hkv, d), 52), rnd_bits((2000, hkv, d), 53)
    k = grown(k, by)
    want, want_lse, tol, tol_lse = S.cross_attention(S.values(q), S.values(k), S.values(v), [queries], [2000], scale)
    got, lse = B.cross_attn(dev_bf16(q), dev_bf16(k), dev_bf16(v), scale, want_lse=True)
    close(host_f64(got), want, tol)
    assert (np.abs(host_f64(lse) - want_lse) <= tol_lse).all()


@pytest.mark.parametrize("heads", [(2, 2, 64), (2, 2, 128)])
def test_a_key_that_makes_up_a_row(B, heads):
    """Where a key has nine tenths of its row's weight and more, the probabilities of its 32 are carried in two bf16: only the other keys' terms are off by one's."""
    hq, hkv, d = heads
    queries, states = 200, 1500
    q, k, v = rnd_bits((queries, hq, d), 67), rnd_bits((states, hkv, d), 68), rnd_bits((states, hkv, d), 69)
    at = 700 + 3 * np.arange(queries)
    scale = d ** -0.5
    k[at] = bits(S.values(q) * 12 / scale / (S.values(q) ** 2).sum(2, keepdims=True))    # a logit of 12, among others of up to 4
    x = np.einsum("qhd,khd->hqk", S.values(q), S.values(k)) * scale
    w = np.exp(x - x.max(2, keepdims=True))
    w /= w.sum(2, keepdims=True)
    own = w[:, np.arange(queries), at]
    assert own.min() > 0.9
    want, _, tol, _ = S.cross_attention(S.values(q), S.values(k), S.values(v), [queries], [states], scale, parts=2)
    w[:, np.arange(queries), at] = 0
    tol += 1.01 * 2.0 ** -8 * np.einsum("hqk,khd->qhd", w, np.abs(S.values(v)))
    close(host_f64(B.cross_attn(dev_bf16(q), dev_bf16(k), dev_bf16(v), scale)), want, tol)


@pytest.mark.parametrize("queries,states", [(2, 90), (2, 700), (60, 90), (60, 700)])
def test_values_whose_sum_is_beyond_32_bits(B, queries, states):
    """All values of two columns are nearly the type's largest: their mean is one of its numbers."""
    q, k, v = rnd_bits((queries, 16, 128), 54), rnd_bits((states, 2, 128), 55), rnd_bits((states, 2, 128), 56)
    v[:, :, 5], v[:, :, 6], v[::2, :, 7], v[1::2, :, 7] = 0x7f70, 0xff70, 0x7f70, 0xff70
    want, _, tol, _ = S.cross_attention(S.values(q), S.values(k), S.values(v), [queries], [states], 0.1)
    close(host_f64(B.cross_attn(dev_bf16(q), dev_bf16(k), dev_bf16(v), 0.1)), want, tol)


@pytest.mark.parametrize("queries,states", [(2, 90), (2, 2700), (60, 90), (60, 2700)])
def test_odd_values_where_the_queries_are_the_output(B, queries, states):
    """A row that is summed once more reads its query once more: rows with one piece and with many."""
    q, k, v = dev_bf16(rnd_bits((queries, 16, 128), 57)), dev_bf16(rnd_bits((states, 2, 128), 58)), dev_bf16(rnd_bits((states, 2, 128), 59))
    v[states // 2, :, 5], v[7, 1, 6] = np.inf, np.nan
    want = B.cross_attn(q, k, v, 0.1)
    assert (want[:, :, 5] == np.inf).all() and want[:, 8:, 6].isnan().all()
    B.cross_attn(q, k, v, 0.1, out=q)
    assert (q.view(torch.int16) == want.view(torch.int16)).all()


def test_ranges_of_many_entries(B):
    """Entries of no query, of some and of more than a share, with states and without, and some that leave the tensors."""
    rng = np.random.default_rng(60)
    n = 700
    q_lens, kv_lens = (rng.integers(0, 4, n) * rng.integers(0, 2, n)).tolist(), (rng.integers(0, 90, n) * rng.integers(0, 2, n)).tolist()
    q_lens[350], kv_lens[350], q_lens[699], kv_lens[699] = 300, 1000, 70, 333
    ranges = np.sort(rng.integers(-9, 120, (sum(q_lens), 2)), axis=1).astype(np.int32)
    at = sum(q_lens[:350])
    ranges[at:at + 300] *= 9
    check_cross(B, 61, (4, 1, 64), q_lens, kv_lens, ranges=ranges)
    cu_q, cu_kv = (np.concatenate([[0], np.cumsum(x)]) for x in (q_lens, kv_lens))
    q, k = dev_bf16(rnd_bits((sum(q_lens), 4, 64), 62)), dev_bf16(rnd_bits((sum(kv_lens), 1, 64), 63))
    want, _, tol, _ = S.cross_attention(host_f64(q), host_f64(k), host_f64(k), q_lens, kv_lens, 0.125, ranges)
    cu_kv[1:200] = sum(kv_lens) + 1                          # (of the entries up to 199)
    out = torch.full_like(q, 7.0)
    B.cross_attn(q, k, k, 0.125, cu_q=i32(cu_q), cu_kv=i32(cu_kv), key_ranges=i32(ranges), out=out)
    assert (out[:cu_q[200]] == 7.0).all()
    # (where a row's states are cut depends on the other entries, so the bits may differ: the bounds hold for every cut)
    close(host_f64(out)[cu_q[200]:], want[cu_q[200]:], tol[cu_q[200]:])


@pytest.mark.parametrize("cu_q,left", [([0, 40, 999, 40, 70], [0, 3]), ([0, 40, -3, 40, 70], [0, 3]), ([5, -9, 0, 40, 70], [2, 3]), ([0, 40, 70, 2 ** 31 - 1, -(2 ** 31)], [0, 1])])
@pytest.mark.parametrize("kind", ["cross", "ranges", "paged"])
def test_entries_that_are_skipped_change_no_other(B, cu_q, left, kind):
    """Offsets that make no entry, in front of and between others whose rows are cut and joined."""
    q, k = rnd_bits((70, 14, 64), 71), rnd_bits((4 * 2000, 2, 64), 72)
    out = torch.full((70, 14, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    ranges = np.stack([np.arange(70) * 20, 1000 + np.arange(70) * 9], 1).astype(np.int32) if kind == "ranges" else None
    pages = k.reshape(4, 125, 16, 2, 64)
    if kind == "paged":
        table = np.arange(500, dtype=np.int32).reshape(4, 125)
        B.shared_attn(dev_bf16(q), dev_bf16(pages.reshape(500, 16, 2, 64)), dev_bf16(pages.reshape(500, 16, 2, 64)), i32(table), i32([2000] * 4), 0.125,
                      torch.zeros((3, 4), dtype=torch.int32, device="cuda"), cu_q=i32(cu_q), max_q_len=40, max_kv_len=2000, out=out)
    else:
        B.cross_attn(dev_bf16(q), dev_bf16(k), dev_bf16(k), 0.125, cu_q=i32(cu_q), cu_kv=i32([0, 2000, 4000, 6000, 8000]),
                     key_ranges=None if ranges is None else i32(ranges), out=out)
    got, written = host_f64(out), np.zeros(70, dtype=bool)
    for e in left:
        rows, x = slice(cu_q[e], cu_q[e + 1]), S.values(k[2000 * e:2000 * e + 2000])
        sees = np.arange(2000)[None] <= 2000 - (cu_q[e + 1] - cu_q[e]) + np.arange(cu_q[e + 1] - cu_q[e])[:, None] if kind == "paged" else None
        if kind == "paged":
            want, _, tol, _ = S.all_heads(S.values(q[rows]), x, x, 0.125, sees)
        else:
            want, _, tol, _ = S.cross_attention(S.values(q[rows]), x, x, [cu_q[e + 1] - cu_q[e]], [2000], 0.125, None if ranges is None else ranges[rows])
        close(got[rows], want, tol)
        written[rows] = True
    assert (got[~written] == 7.0).all()


@pytest.mark.parametrize("ranges", [False, True])
def test_more_heads_of_a_group_than_a_set_has_rows(B, ranges):
    check_cross(B, 73, (300, 1, 64), [3, 2], [100, 700], ranges=np.array([[0, 90], [5, 60], [50, 100], [0, 700], [333, 650]], dtype=np.int32) if ranges else None)
    check(B, *build(74, [(96, [(20, 2), (40, 3)])], (300, 1, 64), 16))


@pytest.mark.parametrize("odd", [False, True])
def test_rows_in_place_and_cut_rows_where_there_are_many(B, odd):
    """More than 2^17 rows: a wave of the join looks at several heads of a token."""
    heads, queries, states = (64, 8, 64), 2100, 190
    q, k, v = rnd_bits((queries, 64, 64), 75), rnd_bits((states, 8, 64), 76), rnd_bits((states, 8, 64), 77)
    flat = v.copy()
    if odd:
        v[100, 3, 7], v[40, 5, 9], flat[100, 3, 7], flat[40, 5, 9] = 0x7f80, 0x7fc0, 0, 0
    want, want_lse, tol, tol_lse = S.cross_attention(S.values(q), S.values(k), S.values(flat), [queries], [states], 0.125)
    got, lse = B.cross_attn(dev_bf16(q), dev_bf16(k), dev_bf16(v), 0.125, want_lse=True)
    got = host_f64(got)
    assert (np.abs(host_f64(lse) - want_lse) <= tol_lse).all()
    plain = np.ones((64, 64), dtype=bool)
    if odd:
        assert (got[:, 24:32, 7] == np.inf).all() and np.isnan(got[:, 40:48, 9]).all()
        plain[24:32, 7] = plain[40:48, 9] = False
    assert (np.abs(got - want)[:, plain] <= tol[:, plain]).all()


def test_many_rows_that_share_keys(B):
    check(B, *build(78, [(64, [(80, 60)] * 36)], (64, 8, 64), 16))


def test_captured_graphs_that_share_a_workspace(B):
    """One after the other, again and again, each with its own answers."""
    one = build(64, [(800, [(20, 2)] * 5)], (14, 2, 64), 16)
    qs, ks, vs = dev_bf16(one[0]), dev_bf16(one[1]), dev_bf16(one[2])
    table, lens, groups = i32(one[3]), i32(one[4]), i32(one[6])
    qc, kc = dev_bf16(rnd_bits((40, 14, 64), 65)), dev_bf16(rnd_bits((900, 2, 64), 66))
    ranges = i32([[t * 5, 700 + t * 3] for t in range(40)])
    bytes_ = max(B.shared_attn_workspace_bytes(5, 10, 14, 2, 64), B.cross_attn_workspace_bytes(1, 40, 14, 2, 64))
    workspace = B.new_workspace(bytes_)
    outs = torch.zeros_like(qs), torch.zeros_like(qc)
    calls = [lambda **kw: B.shared_attn(qs, ks, vs, table, lens, 0.125, groups, **kw), lambda **kw: B.cross_attn(qc, kc, kc, 0.125, key_ranges=ranges, **kw)]
    want = [call() for call in calls]
    graphs = []
    for call, out in zip(calls, outs):
        call(out=out, workspace=workspace)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(out=out, workspace=workspace)
    for _ in range(5):
        for g, out, w in zip(graphs, outs, want):
            out.fill_(3.0)
            g.replay()
            assert (out == w).all()
            calls[1](workspace=workspace)


# ------------------------------------------------------------------------------------------------ who shares
def check_groups(B, table, kv_lens, q_lens, n_pages, ps, min_tokens):
    want = S.groups(np.asarray(table), kv_lens, q_lens, n_pages, ps, min_tokens)
    got = B.pages_shared(i32(table), i32(kv_lens), n_pages, ps, 0, cu_q=i32(np.concatenate([[0], np.cumsum(q_lens)])), min_tokens=min_tokens)
    assert (got.cpu().numpy() == want).all(), (got.cpu().numpy(), want)
    if len(set(q_lens)) == 1:
        again = B.pages_shared(i32(table), i32(kv_lens), n_pages, ps, q_lens[0], min_tokens=min_tokens)
        assert (again.cpu().numpy() == want).all()
    return want


@pytest.mark.parametrize("min_tokens", [0, 1, 100, 5000])
@pytest.mark.parametrize("ps", [16, 48])
def test_who_shares(B, ps, min_tokens):
    args = build(3, [(ps * 20, [(9, 3), (30, 1)]), (0, [(1, 1)]), (0, [(150, 2)]), (ps * 7, [(5, 5), (80, 40), (16, 1)]), (ps, [(2, 2), (1, 1)])], (1, 1, 64), ps)
    _, k, _, table, kv_lens, q_lens, groups = args
    got = check_groups(B, table, kv_lens, q_lens, len(k), ps, min_tokens)
    if min_tokens <= 1:
        assert (got == groups).all()


@pytest.mark.parametrize("batch,width", [(1, 1), (2, 1), (3, 300), (40, 70), (257, 9), (1500, 5), (9, 3000), (16, 512), (16, 513), (17, 512), (8, 256), (5, 257)])
@pytest.mark.parametrize("seed", [1, 2])
def test_who_shares_in_tables_of_every_kind(B, batch, width, seed):
    """Rows that go on from the row before them at a random place; entries that are no pages; blocks longer than their caches."""
    rng = np.random.default_rng((batch, width, seed))
    table = rng.integers(0, 50, (batch, width)).astype(np.int32)
    for b in range(1, batch):
        n = int(rng.integers(0, width + 1)) if rng.random() < 0.8 else width
        table[b, :n] = table[b - 1, :n]
    table[rng.random((batch, width)) < 0.3 / width] = [-1, 50, -(2 ** 31), 2 ** 31 - 1][seed % 4]
    kv_lens = rng.integers(0, width * 16 + 1, batch) if seed == 1 else rng.integers(max(0, width * 16 - 20), width * 16 + 200, batch)
    q_lens = rng.integers(0, 12, batch)
    check_groups(B, table, kv_lens.tolist(), q_lens.tolist(), 50, 16, int(rng.choice([0, 16, 64])))


def test_nested_prefixes(B):
    """Two videos behind one instruction are two groups; all of them one where there is no more than the instruction."""
    table = np.arange(6 * 40).reshape(6, 40)
    table[:, :4] = table[0, :4]
    two = table.copy()
    two[1:3, :30] = two[0, :30]
    two[4:, :25] = two[3, :25]
    assert check_groups(B, two, [600] * 6, [1] * 6, 240, 16, 1).tolist() == [[0, 0, 0, 3, 3, 3], [3, 0, 0, 3, 0, 0], [480] * 3 + [400] * 3]
    assert check_groups(B, table, [600] * 6, [1] * 6, 240, 16, 1).tolist() == [[0] * 6, [6, 0, 0, 0, 0, 0], [64] * 6]


# ------------------------------------------------------------------------------------------------ together, streams, graphs
def test_from_forks_to_attention(B):
    """One video, four questions: forked, grown, found, turned and written, attended to; then a step on; as if each had a cache of its own."""
    torch.manual_seed(5)
    ps, d, hq, hkv, n_pages = 16, 64, 4, 2, 64
    k, v = (torch.randn(n_pages, ps, hkv, d, device="cuda").bfloat16() for _ in range(2))
    turns = B.rope_turns(d, 1e4)
    table = torch.full((1, 24), -1, dtype=torch.int32, device="cuda")
    # the video's 200 tokens
    table = B.pages_assign(table, i32([-1]), i32([0]), i32([200]), n_pages, ps)[0]
    lens, q_len = [200] * 4, 6
    parent, keep = i32([0] * 4), i32([200] * 4)
    for step in range(3):
        lens = [n + q_len for n in lens]
        old = table
        table, start, rows, refs, status = B.pages_assign(old, parent, keep, i32(lens), n_pages, ps)
        assert status.tolist() == [0] * 4
        B.pages_copy(k[None], v[None], old, k[None], v[None], table, rows, ps, src_row=parent, src_start=start, dst_start=start)
        groups = B.pages_shared(table, i32(lens), n_pages, ps, q_len, min_tokens=16)
        assert groups.tolist() == [[0] * 4, [4, 0, 0, 0], [192] * 4]
        q, kn, vn = (torch.randn(4 * q_len, h, d, device="cuda").bfloat16() for h in (hq, hkv, hkv))
        q = B.rope_append(kn, vn, k, v, table, i32(lens), q=q, turns=turns)
        got = B.shared_attn(q, k, v, table, i32(lens), 0.125, groups)
        want = B.paged_attn(q, k, v, table, i32(lens), 0.125)
        plain, _, tol, _, _ = S.shared_attention(host_f64(q), host_f64(k), host_f64(v), table.cpu().numpy(), lens, [q_len] * 4, 0.125)
        close(host_f64(got), plain, tol)
        close(host_f64(want), plain, tol)
        parent, keep = i32([0, 1, 2, 3]), i32(lens)


def test_a_layer_over_caches_and_states(B):
    """Questions about two videos: who shares, attention over their caches, then over the states of each one's encoder, in place."""
    q, k, v, table, kv_lens, q_lens, groups = build(84, [(320, [(20, 3), (35, 1), (50, 4)]), (160, [(60, 2), (16, 5)])], (16, 2, 128), 16)
    states = [300, 1100]
    ks, vs = rnd_bits((sum(states), 2, 128), 85), rnd_bits((sum(states), 2, 128), 86)
    cu_q, lens = i32(np.concatenate([[0], np.cumsum(q_lens)])), i32(kv_lens)
    found = B.pages_shared(i32(table), lens, len(k), 16, max(q_lens), cu_q=cu_q, min_tokens=16)
    assert found.tolist() == groups.tolist()
    x = B.shared_attn(dev_bf16(q), dev_bf16(k), dev_bf16(v), i32(table), lens, 0.1, found, cu_q=cu_q, max_q_len=max(q_lens))
    want, _, tol, _, _ = S.shared_attention(S.values(q), S.values(k), S.values(v), table, kv_lens, q_lens, 0.1)
    close(host_f64(x), want, tol)
    texts = [sum(q_lens[:3]), sum(q_lens[3:])]
    want, _, tol, _ = S.cross_attention(host_f64(x), S.values(ks), S.values(vs), texts, states, 0.1)
    out = B.cross_attn(x, dev_bf16(ks), dev_bf16(vs), 0.1, cu_q=i32([0, texts[0], sum(texts)]), cu_kv=i32([0, states[0], sum(states)]), out=x)
    assert out is x
    close(host_f64(x), want, tol)


def test_a_captured_step_while_groups_and_lengths_change(B):
    ps, heads = 16, (4, 1, 64)
    one = build(21, [(320, [(20, 2)] * 3), (0, [(30, 2)])], heads, ps)
    two = build(22, [(0, [(330, 2)]), (160, [(20, 2)] * 2), (0, [(60, 2)])], heads, ps)
    pool_k, pool_v = (rnd_bits(one[1].shape, i) for i in (25, 26))    # (the second table names pages that the first has no rows in)
    q, k, v = dev_bf16(one[0]), dev_bf16(pool_k), dev_bf16(pool_v)
    table, lens = i32(one[3]), i32(one[4])
    pages = len(one[1])
    groups = torch.zeros((3, 4), dtype=torch.int32, device="cuda")
    workspace, scratch = B.new_workspace(B.shared_attn_workspace_bytes(4, 8, *heads)), B.new_workspace(B.pages_shared_workspace_bytes(4))
    out = torch.zeros_like(q)

    def step():
        B.pages_shared(table, lens, pages, ps, 2, min_tokens=1, groups=groups, workspace=scratch)
        return B.shared_attn(q, k, v, table, lens, 0.125, groups, out=out, want_lse=True, workspace=workspace)[1]

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lse = step()
    width = table.shape[1]
    for turn in range(4):
        q_, k_, v_, t_, n_, _, g_ = (one, two)[turn % 2]
        rows = np.full((4, width), -1, dtype=np.int32)
        rows[:, :t_.shape[1]] = t_[:, :width]
        rows = np.where(rows < pages, rows, -1)
        q.copy_(dev_bf16(q_))
        table.copy_(i32(rows))
        lens.copy_(i32(n_))
        graph.replay()
        torch.cuda.synchronize()
        got, got_lse = out.clone(), lse.clone()
        eager = B.shared_attn(q, k, v, table, lens, 0.125, B.pages_shared(table, lens, pages, ps, 2, min_tokens=1), want_lse=True)
        assert (got == eager[0]).all() and (got_lse == eager[1]).all()
        want, _, tol, _, _ = S.shared_attention(S.values(q_), S.values(pool_k), S.values(pool_v), rows, n_, [2] * 4, 0.125)
        close(host_f64(got), want, tol)


def test_the_same_call_gives_the_same_bits_on_other_streams(B):
    args = build(23, [(800, [(20, 3)] * 9)], (28, 4, 128), 16)
    q, k, v, table, kv_lens, q_lens, groups = args
    dev = dev_bf16(q), dev_bf16(k), dev_bf16(v), i32(table), i32(kv_lens), 0.1, i32(groups)
    want = B.shared_attn(*dev)
    states = dev[1].flatten(0, 1)
    finite = torch.where(torch.isfinite(states), states, torch.zeros_like(states))
    cross = B.cross_attn(dev[0], finite, finite, 0.1)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(3)], []
    for s in streams:
        with torch.cuda.stream(s):
            got.append((B.shared_attn(*dev), B.cross_attn(dev[0], finite, finite, 0.1)))
    torch.cuda.synchronize()
    for a, b in got:
        assert (a == want).all() and (b == cross).all()


def test_workspaces_may_hold_anything(B):
    args = build(24, [(800, [(20, 3)] * 4)], (14, 2, 64), 16)
    q, k, v, table, kv_lens, q_lens, groups = args
    want = check(B, *args)
    for fill in (0x00, 0x7f, 0xff):
        w = B.new_workspace(B.shared_attn_workspace_bytes(4, 12, 14, 2, 64)).fill_(fill)
        got = B.shared_attn(dev_bf16(q), dev_bf16(k), dev_bf16(v), i32(table), i32(kv_lens), 0.125, i32(groups), workspace=w)
        assert (host_f64(got) == want).all()


@pytest.mark.skipif(torch.cuda.device_count() < 1, reason="no GPU")
def test_caches_beyond_32_bits(B):
    """Pages whose bytes lie more than 4 GiB into the pool, and states that do."""
    ps, hkv, d = 64, 8, 128
    pages = 40000                                            # 5.2 GB of keys
    k = torch.zeros((pages, ps, hkv, d), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    far = [39999, 39000, 35001, 5, 38888]
    for i, page in enumerate(far):
        k[page] = dev_bf16(rnd_bits((ps, hkv, d), (31, i)))
        v[page] = dev_bf16(rnd_bits((ps, hkv, d), (32, i)))
    table = np.array([far[:4], far[:3] + far[4:]], dtype=np.int32)
    q = dev_bf16(rnd_bits((4, 64, d), 33))
    groups = i32([[0, 0], [2, 0], [192, 192]])
    got = B.shared_attn(q, k, v, i32(table), i32([250, 230]), 0.1, groups)
    small = [x[far] for x in (k, v)]
    want = B.shared_attn(q, *small, i32([[0, 1, 2, 3], [0, 1, 2, 4]]), i32([250, 230]), 0.1, groups)
    assert (got == want).all()
    flat_k, flat_v = k.view(-1, hkv, d), v.view(-1, hkv, d)
    at = 39999 * ps
    got = B.cross_attn(q, flat_k, flat_v, 0.1, cu_q=i32([0, 0, 4]), cu_kv=i32([0, at, at + ps]))
    assert (got == B.cross_attn(q, flat_k[at:], flat_v[at:], 0.1)).all()
