"""Attention over the MXFP4 cache against a 64-bit form: head widths, groups,
pages, lengths around the kernels' tiles, masks that leave rows empty, ragged
batches, splits of the tokens over workgroups, and what may stand in unused places."""
import numpy as np
import pytest
import torch

import paper_2608_26581_amd as rfq
import kv_util as ku

pytestmark = pytest.mark.gpu


def _starts(reqs):
    return np.concatenate(([0], np.cumsum([q for _, q in reqs]))).astype(np.int32)


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _queries(rng, T, Hq, D):
    return ku.bf16(rng.standard_normal((T, Hq, D)))


def _run(q, cache, reqs, causal=True, window=0, scale=None, **kw):
    lens = np.array([n for n, _ in reqs], np.int32)
    return rfq.rfq_kv_attention(
        _dev(q.astype(np.float32)).bfloat16(), cache.device(), _dev(cache.tables), _dev(lens),
        _dev(_starts(reqs)), max([1] + [n for _, n in reqs]), max([1] + [n for n, _ in reqs]),
        scale=scale, causal=causal, window=window, return_lse=True, **kw)


def _check(rng, reqs, Hq, heads, D, page, causal=True, window=0, scale=None, **kw):
    lens = [n for n, _ in reqs]
    cache = ku.Cache(rng, lens, heads, page, D)
    q = _queries(rng, int(_starts(reqs)[-1]), Hq, D)
    print("attention %s Hq=%d heads=%d D=%d page=%d causal=%s window=%d" % (
        reqs[:6], Hq, heads, D, page, causal, window), flush=True)
    out, lse = _run(q, cache, reqs, causal, window, scale, **kw)
    ref = ku.attention(q, cache, lens, _starts(reqs), D ** -0.5 if scale is None else scale,
                       causal, window)
    torch.cuda.synchronize()
    ku.assert_attention_close(out.float().cpu().numpy(), lse.cpu().numpy(), ref, str(reqs[:4]))
    return cache, q, out, lse


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("group", [1, 5, 8, 16, 20])
def test_decode_lengths(D, page, group):
    rng = np.random.default_rng(D + page + group)
    reqs = [(n, 1) for n in (1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 200, 255, 256)]
    _check(rng, reqs, 2 * group, 2, D, page)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("length", [257, 300, 1000, 5003])
def test_decode_split(D, length):
    rng = np.random.default_rng(length + D)
    _check(rng, [(length, 1)], 8, 2, D, 16)
    _check(rng, [(length, 1), (7, 1), (0, 0), (length // 3, 1), (0, 1)], 6, 1, D, 64)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("group", [1, 4, 7])
@pytest.mark.parametrize("causal", [True, False])
def test_several_queries(D, group, causal):
    rng = np.random.default_rng(D + group)
    reqs = [(3, 3), (70, 5), (300, 17), (0, 0), (64, 64), (129, 33), (400, 1)]
    _check(rng, reqs, 2 * group, 2, D, 32, causal=causal)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("nq", [65, 130, 257])
@pytest.mark.parametrize("extra", [0, 1, 100, 191])
@pytest.mark.parametrize("causal", [True, False])
def test_prompts(D, nq, extra, causal):
    rng = np.random.default_rng(D + nq + extra)
    _check(rng, [(nq + extra, nq)], 4, 1, D, 64, causal=causal)


# Enough row tiles that requests of more than a few rows take the kernel of 128-row
# workgroups: 64 heads with two queries each, about 150 rows of q.
WIDE = [[(150, 150)], [(171, 70), (64, 64), (33, 1), (90, 40)], [(40, 40), (0, 0), (2, 2), (129, 128)],
        [(65, 64), (0, 3), (20, 90)]]


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("reqs", WIDE)
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 37), (False, 70)])
def test_many_rows(D, reqs, causal, window):
    rng = np.random.default_rng(D + window)
    _check(rng, reqs, 128, 64, D, 16, causal=causal, window=window)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 700, 1500])
@pytest.mark.parametrize("causal", [True, False])
def test_many_rows_split(D, window, causal):
    """Few row tiles over long histories: the tokens in parts, some of them empty."""
    rng = np.random.default_rng(D + window)
    _check(rng, [(4600, 40), (2500, 1), (2100, 70), (0, 33), (30, 30)], 8, 2, D, 64, causal=causal,
           window=window)
    _check(rng, [(3000, 20)], 10, 2, D, 16, causal=causal, window=window)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("nq", [1, 7])
@pytest.mark.parametrize("B,longest", [(6, 1024), (6, 1025), (270, 200), (270, 290)])
@pytest.mark.parametrize("window", [0, 90])
def test_whole_and_split_items(D, nq, B, longest, window):
    """Both sides of the rules on items and tokens, one and several rows a request."""
    rng = np.random.default_rng(D + nq + B + longest)
    reqs = [(longest, nq)] + [(int(n), int(rng.integers(0, nq + 1)))
                              for n in rng.integers(0, longest, B - 1)]
    _check(rng, reqs, 6, 2, D, 16, window=window)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("length", [255, 511, 512, 513, 800, 1027])
def test_many_rows_short_parts(D, length):
    rng = np.random.default_rng(length)
    _check(rng, [(length, 70)], 2, 2, D, 32)
    _check(rng, [(length, 67), (300, 10), (0, 70)], 2, 1, D, 16, causal=False, window=400)


@pytest.mark.parametrize("group,heads,page", [(1, 128, 32), (3, 48, 128), (7, 20, 64), (20, 8, 256)])
def test_many_rows_groups(group, heads, page):
    rng = np.random.default_rng(group)
    _check(rng, [(200, 110), (70, 40)], group * heads, heads, 64, page)


@pytest.mark.parametrize("scale", [25.0, -0.7, 0.0])
def test_many_rows_scale(scale):
    rng = np.random.default_rng(17)
    _check(rng, [(180, 130), (20, 20)], 128, 64, 64, 16, scale=scale)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_many_rows_missing_and_nan_blocks(D):
    """Table entries outside the cache, and NaN blocks reaching only rows that attend."""
    rng = np.random.default_rng(18)
    reqs = [(220, 130), (60, 20)]
    cache = ku.Cache(rng, [n for n, _ in reqs], 64, 16, D)
    cache.tables[0, 2] = -1
    cache.tables[0, 11:13] = 2 ** 31 - 1
    for token, part, head in ((100, 1, 3), (160, 3, 7), (170, 3, 3), (30, 1, 9)):
        cache.parts[part][cache.tables[0, token // 16], head, token % 16, D // 64] = 255
    q = _queries(rng, 150, 128, D)
    for window in (0, 60):
        out, lse = _run(q, cache, reqs, window=window)
        ref = ku.attention(q, cache, [n for n, _ in reqs], _starts(reqs), D ** -0.5, True, window)
        nan = np.isnan(ref[0]).any(-1)
        got = out.float().cpu().numpy()
        assert np.array_equal(np.isnan(got).all(-1), nan) and np.array_equal(np.isnan(got).any(-1), nan)
        tol = (2.0 ** -8 + 2.0 ** -15 * ref[3][..., None]) * ref[2] + 2.0 ** -8 * np.abs(ref[0])
        assert np.all((np.abs(got - ref[0]) <= tol)[~nan])


def test_long_prompt_over_many_workgroups():
    """Enough rows that the row tiles alone fill the GPU."""
    rng = np.random.default_rng(5)
    _check(rng, [(700, 600), (513, 450), (90, 90)], 32, 8, 64, 32)
    _check(rng, [(530, 500), (300, 280)], 28, 4, 128, 16, window=200)


@pytest.mark.parametrize("window", [1, 2, 16, 63, 64, 65, 300, 5000])
@pytest.mark.parametrize("causal", [True, False])
def test_window(window, causal):
    rng = np.random.default_rng(window)
    _check(rng, [(700, 1), (130, 40), (64, 64), (1, 1), (65, 2)], 4, 2, 64, 16, causal=causal,
           window=window)
    _check(rng, [(900, 150), (40, 1)], 4, 1, 128, 64, causal=causal, window=window)


def test_rows_without_tokens():
    """More queries than tokens (rows before the first token), no tokens at all, and a
    request without queries."""
    rng = np.random.default_rng(3)
    for causal in (True, False):
        _, _, out, lse = _check(rng, [(0, 3), (2, 5), (5, 0), (1, 1), (0, 130), (3, 140)], 4, 2, 64,
                                16, causal=causal)
        assert torch.all(out[:3] == 0) and torch.all(torch.isneginf(lse[:3]))


def test_many_requests():
    """More requests than a workgroup has threads, most of them short."""
    rng = np.random.default_rng(4)
    reqs = [(int(n), 1) for n in rng.integers(0, 90, 700)]
    reqs[350] = (1500, 1)
    reqs[351] = (40, 3)
    _check(rng, reqs, 4, 2, 64, 16)


def test_blocks_missing_from_the_table():
    rng = np.random.default_rng(6)
    reqs = [(300, 1), (200, 20), (130, 1), (260, 90)]
    cache = ku.Cache(rng, [n for n, _ in reqs], 2, 16, 128)
    cache.tables[0, 3] = -1
    cache.tables[0, 7:9] = cache.blocks
    cache.tables[1, 0] = 2 ** 31 - 1
    cache.tables[2, :] = -5
    cache.tables[3, 1:6] = -1
    q = _queries(rng, 112, 8, 128)
    out, lse = _run(q, cache, reqs)
    ref = ku.attention(q, cache, [n for n, _ in reqs], _starts(reqs), 128 ** -0.5, True, 0)
    torch.cuda.synchronize()
    ku.assert_attention_close(out.float().cpu().numpy(), lse.cpu().numpy(), ref)
    assert torch.all(out[21] == 0)


def test_lengths_beyond_the_table():
    """A length that the table cannot hold is cut to it."""
    rng = np.random.default_rng(7)
    cache = ku.Cache(rng, [64, 32], 1, 16, 64, width=4)
    q = _queries(rng, 3, 4, 64)
    out, lse = rfq.rfq_kv_attention(
        _dev(q.astype(np.float32)).bfloat16(), cache.device(), _dev(cache.tables),
        _dev(np.array([2 ** 31 - 1, 32], np.int32)), _dev(np.array([0, 2, 3], np.int32)), 2, 64,
        return_lse=True)
    ref = ku.attention(q, cache, [64, 32], [0, 2, 3], 0.125, True, 0)
    torch.cuda.synchronize()
    ku.assert_attention_close(out.float().cpu().numpy(), lse.cpu().numpy(), ref)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("reqs", [[(100, 1), (90, 1)], [(600, 1), (500, 1)],
                                  [(150, 100), (140, 140)]])
def test_nan_blocks_reach_only_rows_that_attend(D, reqs):
    """Key and value blocks with the NaN scale make NaN of the rows that attend to
    their token, and nothing of the others (causal, window, other requests)."""
    rng = np.random.default_rng(8)
    cache = ku.Cache(rng, [n for n, _ in reqs], 2, 16, D)
    T = sum(n for _, n in reqs)
    q = _queries(rng, T, 4, D)
    n, nq = reqs[0]
    for token, part, head in ((n - nq // 2 - 1, 1, 0), (n - 1 - nq // 3, 3, 1), (0, 3, 0)):
        block, off = cache.tables[0, token // 16], token % 16
        cache.parts[part][block, head, off, D // 32 - 1] = 255
    for window in (0, 3, 40):
        out, lse = _run(q, cache, reqs, window=window)
        ref = ku.attention(q, cache, [n for n, _ in reqs], _starts(reqs), D ** -0.5, True, window)
        ref_nan = np.isnan(ref[0]).any(-1)
        got = out.float().cpu().numpy()
        assert np.array_equal(np.isnan(got).all(-1), ref_nan), window
        assert np.array_equal(np.isnan(got).any(-1), ref_nan), window
        ok = ~ref_nan
        tol = (2.0 ** -8 + 2.0 ** -15 * ref[3][..., None]) * ref[2] + 2.0 ** -8 * np.abs(ref[0])
        assert np.all((np.abs(got - ref[0]) <= tol)[ok]), window


@pytest.mark.parametrize("fill", [0, 128, 252, 253, 254, 255])
def test_unused_places_have_no_influence(fill):
    """The same bits whatever unused tokens, blocks and rows hold."""
    rng = np.random.default_rng(9)
    reqs = [(37, 1), (300, 1), (200, 130), (5, 5)]
    cache = ku.Cache(rng, [n for n, _ in reqs], 2, 64, 128)
    q = _queries(rng, 137, 8, 128)
    ref = _run(q, cache, reqs)
    for part in (1, 3):
        unused = cache.parts[part] == 255
        cache.parts[part][unused] = fill
        cache.parts[part - 1][np.repeat(unused, 16, -1)] ^= 0x5A
    got = _run(q, cache, reqs)
    for a, b in zip(ref, got):
        assert torch.equal(a, b)


def test_large_scores_and_scale():
    """Scores far apart (all but one P vanish) and a negative scale."""
    rng = np.random.default_rng(10)
    for scale in (30.0, -2.0, 0.0):
        _check(rng, [(500, 2), (33, 33)], 4, 2, 64, 16, scale=scale)


def test_strided_queries_and_output():
    """q as a slice of a joint projection, out as a slice of a wider tensor; nothing
    beside the rows is written."""
    rng = np.random.default_rng(11)
    reqs = [(90, 3), (300, 1), (150, 60)]
    cache = ku.Cache(rng, [n for n, _ in reqs], 2, 16, 128)
    q = _queries(rng, 66, 8, 128)                         # two rows of padding
    joint = torch.full((66, 12, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    joint[:, :8] = _dev(q.astype(np.float32)).bfloat16()
    wide = torch.full((66, 10, 136), 7.0, dtype=torch.bfloat16, device="cuda")
    lens = np.array([n for n, _ in reqs], np.int32)
    args = (cache.device(), _dev(cache.tables), _dev(lens), _dev(_starts(reqs)), 60, 300)
    out, lse = rfq.rfq_kv_attention(joint[:, :8], *args, return_lse=True, out=wide[:, 1:9, :128])
    ref = ku.attention(q[:64], cache, lens, _starts(reqs), 128 ** -0.5, True, 0)
    torch.cuda.synchronize()
    ku.assert_attention_close(out[:64].float().cpu().numpy(), lse[:64].cpu().numpy(), ref)
    untouched = wide.clone()
    untouched[:64, 1:9, :128] = 7.0
    assert torch.all(untouched == 7.0)
    # Heads before tokens in memory.
    turned = joint[:, :8].transpose(0, 1).contiguous().transpose(0, 1)
    again = rfq.rfq_kv_attention(turned, *args)
    assert torch.equal(again[:64], out[:64])


def test_workspace_and_bounds():
    """Without a workspace the tokens are not split; a too small hint costs time
    only; a workspace is not read before it is written."""
    rng = np.random.default_rng(12)
    reqs = [(3000, 1), (2000, 2)]
    cache = ku.Cache(rng, [n for n, _ in reqs], 2, 32, 128)
    q = _queries(rng, 3, 8, 128)
    ref = ku.attention(q, cache, [n for n, _ in reqs], _starts(reqs), 128 ** -0.5, True, 0)
    lens = np.array([n for n, _ in reqs], np.int32)
    args = (_dev(q.astype(np.float32)).bfloat16(), cache.device(), _dev(cache.tables), _dev(lens),
            _dev(_starts(reqs)))
    need = rfq.rfq_kv_attention_workspace_bytes(3, 8, 2, 128, 2, 2, 3000)
    assert need > 0
    for fill, nbytes in ((0, need), (255, need), (0x7F, need), (0, need - 16), (0, 0)):
        ws = torch.full((max(nbytes, 16) + 64,), fill, dtype=torch.uint8, device="cuda")
        out, lse = rfq.rfq_kv_attention(*args, 2, 3000, return_lse=True, workspace=ws[:nbytes])
        ku.assert_attention_close(out.float().cpu().numpy(), lse.cpu().numpy(), ref, str(nbytes))
        assert torch.all(ws[nbytes:] == fill)
    out, lse = rfq.rfq_kv_attention(*args, 0, 1, return_lse=True)
    ku.assert_attention_close(out.float().cpu().numpy(), lse.cpu().numpy(), ref)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("reqs", [[(3000, 1), (0, 0), (700, 2)], [(900, 40), (2000, 1)]])
@pytest.mark.parametrize("hint", [2 ** 21, 2 ** 62])
def test_hints_beyond_the_lengths(D, reqs, hint):
    """Upper bounds far above the lengths choose how the work is divided, nothing else."""
    rng = np.random.default_rng(D)
    lens = [n for n, _ in reqs]
    cache = ku.Cache(rng, lens, 2, 16, D)
    starts = _starts(reqs)
    q = _queries(rng, int(starts[-1]), 8, D)
    out, lse = rfq.rfq_kv_attention(
        _dev(q.astype(np.float32)).bfloat16(), cache.device(), _dev(cache.tables),
        _dev(np.array(lens, np.int32)), _dev(starts), 40, hint, return_lse=True)
    ref = ku.attention(q, cache, lens, starts, D ** -0.5, True, 0)
    ku.assert_attention_close(out.float().cpu().numpy(), lse.cpu().numpy(), ref, str(reqs))


def test_same_bits_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(13)
    reqs = [(1500, 1), (40, 1), (700, 1)]
    cache = ku.Cache(rng, [n for n, _ in reqs], 2, 16, 128)
    q = _dev(_queries(rng, 3, 16, 128).astype(np.float32)).bfloat16()
    lens = _dev(np.array([n for n, _ in reqs], np.int32))
    dev_cache, tables, starts = cache.device(), _dev(cache.tables), _dev(_starts(reqs))
    ws = torch.empty(rfq.rfq_kv_attention_workspace_bytes(3, 16, 2, 128, 3, 1, 1500),
                     dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)

    def call():
        return rfq.rfq_kv_attention(q, dev_cache, tables, lens, starts, 1, 1500, out=out,
                                    workspace=ws)
    ref = call().clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = rfq.rfq_kv_attention(q, dev_cache, tables, lens, starts, 1, 1500)
    s.synchronize()
    assert torch.equal(ref, got)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in range(3):
        lens.copy_(_dev(np.array([1500 - 100 * i, 40 - i, 700 - 64 * i], np.int32)))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        assert torch.equal(replayed, call())


def test_offsets_beyond_32_bits():
    """A cache whose codes pass 4 GiB: blocks at its end."""
    heads, page, D = 8, 256, 256
    blocks = (1 << 32) // (heads * page * D // 2) + 40
    cache = rfq.kv_cache(blocks, heads, page, D)
    rng = np.random.default_rng(14)
    small = ku.Cache(rng, [600], heads, page, D, spare=0)
    ids = np.array([blocks - 1, blocks - 30, blocks - 17], np.int32)
    for big, part in zip(cache, small.parts):
        big[torch.from_numpy(ids).long().cuda()] = _dev(part[small.tables[0]])
    q = _queries(rng, 2, 8, D)
    out, lse = rfq.rfq_kv_attention(
        _dev(q.astype(np.float32)).bfloat16(), cache, _dev(ids[None]),
        _dev(np.array([600], np.int32)), _dev(np.array([0, 2], np.int32)), 2, 600, return_lse=True)
    ref = ku.attention(q, small, [600], [0, 2], D ** -0.5, True, 0)
    torch.cuda.synchronize()
    ku.assert_attention_close(out.float().cpu().numpy(), lse.cpu().numpy(), ref)


def test_refusals():
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    cache = rfq.kv_cache(3, 2, 16, 64)
    t = torch.zeros((1, 2), dtype=torch.int32, device="cuda")
    n = torch.ones(1, dtype=torch.int32, device="cuda")
    s = torch.tensor([0, 2], dtype=torch.int32, device="cuda")
    with pytest.raises(TypeError, match="bfloat16"):
        rfq.rfq_kv_attention(q.float(), cache, t, n, s, 2, 16)
    with pytest.raises(ValueError, match="channels"):
        rfq.rfq_kv_attention(q[..., :32], cache, t, n, s, 2, 16)
    with pytest.raises(ValueError, match="contiguous"):
        rfq.rfq_kv_attention(q.transpose(1, 2), cache, t, n, s, 2, 16)
    with pytest.raises(ValueError, match="query_starts"):
        rfq.rfq_kv_attention(q, cache, t, n, s[:1], 2, 16)
    with pytest.raises(ValueError, match="seq_lens"):
        rfq.rfq_kv_attention(q, cache, t, s, s, 2, 16)
    with pytest.raises(TypeError, match="int32"):
        rfq.rfq_kv_attention(q, cache, t.long(), n, s, 2, 16)
    with pytest.raises(ValueError, match="device tensor"):
        rfq.rfq_kv_attention(q, cache, t, n.cpu(), s, 2, 16)
    with pytest.raises(ValueError, match="shape"):
        rfq.rfq_kv_attention(q, cache[:3] + (cache[3][:2],), t, n, s, 2, 16)
    with pytest.raises(rfq.RfqError, match="SHAPE"):
        rfq.rfq_kv_attention(q[:, :3], cache, t, n, s, 2, 16)          # 3 heads over 2
    with pytest.raises(rfq.RfqError, match="SHAPE"):
        rfq.rfq_kv_attention(q, cache, t, n, s, 2, 16, window=-1)
    with pytest.raises(rfq.RfqError, match="SHAPE"):
        rfq.rfq_kv_attention(q, rfq.kv_cache(3, 2, 24, 64), t, n, s, 2, 16)
    with pytest.raises(rfq.RfqError, match="ALIGN"):
        rfq.rfq_kv_attention(torch.zeros(2 * 4 * 64 + 1, dtype=torch.bfloat16,
                                         device="cuda")[1:].view(2, 4, 64), cache, t, n, s, 2, 16)
    assert rfq.rfq_kv_attention(q[:0], cache, t, n, s, 2, 16).shape == (0, 4, 64)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_scale_zero_of_large_scores(D):
    """At scale 0 every token weighs the same, however large its product is."""
    rng = np.random.default_rng(19)
    reqs = [(150, 120), (40, 1)]
    cache = ku.Cache(rng, [n for n, _ in reqs], 2, 16, D)
    q = _queries(rng, 121, 4, D) * 2.0 ** 120
    out, lse = _run(q, cache, reqs, scale=0.0)
    ref = ku.attention(q, cache, [n for n, _ in reqs], _starts(reqs), 0.0, True, 0)
    ku.assert_attention_close(out.float().cpu().numpy(), lse.cpu().numpy(), ref)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n,nq,group", [(5003, 1, 1), (5003, 1, 4), (5003, 3, 8), (5003, 70, 2),
                                        (20011, 1, 4), (20011, 40, 4), (1000, 1, 4), (1024, 9, 2)])
def test_no_token_is_lost(D, n, nq, group):
    """In each head one token's score stands 48 or more above the others', which are 0: each
    row is that token's value, but for its weight's rounding and the result's to bf16
    (2^-9 each) and the others' weights (2^15 2^-69 of at most 3 each together).  The tokens lie at
    the ends of tiles, pages and parts."""
    heads, page = 24, 32
    rng = np.random.default_rng(n + nq)
    cache = ku.Cache(rng, [n], heads, page, D)
    at = [0, 1, 15, 16, 31, 32, 63, 64, 65, n // 3, n // 2, n - nq, n - nq - 1, n // 64 * 64 - 1,
          n // 64 * 64 - 64, n // 256 * 256 - 1, 255, 256, 511, 512]
    at = [min(max(j, 0), n - nq) for j in at] + [int(j) for j in rng.integers(0, n - nq + 1, heads - len(at))]
    cache.parts[0][:] = 0
    cache.parts[1][cache.parts[1] != 255] = 127
    for h, j in enumerate(at):
        cache.parts[0][cache.tables[0, j // page], h, j % page] = 0x77                  # 6 in every channel
    q = np.ones((nq, heads * group, D))
    out, lse = _run(q, cache, [(n, nq)])
    want = np.stack([cache.values(0, h, n)[1][j] for h, j in enumerate(at)])
    want = np.broadcast_to(np.repeat(want, group, 0), (nq, heads * group, D))
    off = np.abs(out.float().cpu().numpy() - want)
    assert np.all(off <= (2.0 ** -8 + 2.0 ** -16) * np.abs(want) + 2.0 ** -50)
    assert np.allclose(lse.cpu().numpy(), 6 * D ** 0.5, rtol=2.0 ** -20, atol=0)
