"""Workspace sizes of the operators at the ends of a model (no GPU): a buffer sized for the largest batch has to
serve every smaller one, so no size may fall as a batch grows."""
import pytest

from paper_2609_37842_amd import eogp as E


def steps(most):
    """Every length up to 5,000, then the neighbourhoods of multiples of 64 (chunks and tiles end there)."""
    out = set(range(1, min(most, 5000) + 1))
    for k in range(5000 // 64, most // 64 + 1):
        out.update((64 * k, 64 * k + 1))
    return sorted(out)


def assert_rising(size, values):
    last = 0
    for v in values:
        got = size(v)
        assert got >= last, (v, got, last)
        last = got


@pytest.mark.parametrize("d", [1, 7, 64, 256, 257, 512, 513, 768, 1024, 1025, 2048, 5121, 16384])
def test_embed_backward_size_rises_with_rows(d):
    assert_rising(lambda n: E.eogp_embed_backward_workspace_size(n, 50257, d), steps(300_000))


@pytest.mark.parametrize("n", [1, 100, 2048, 2049, 6144, 6145, 23808, 65472, 65473, 131009, 262144])
def test_embed_backward_size_rises_with_width_and_vocabulary(n):
    assert_rising(lambda d: E.eogp_embed_backward_workspace_size(n, 50257, d), range(1, 8300))
    assert_rising(lambda V: E.eogp_embed_backward_workspace_size(n, V, 768), range(1, 140_000, 13))


@pytest.mark.parametrize("n,d,chunk", [(1, 1, 8), (2048, 768, 8), (2049, 768, 32), (6145, 2048, 32), (65472, 2048, 32),
                                       (65473, 2048, 64), (262144, 2048, 64), (4_000_000, 64, 64)])
def test_embed_backward_size_holds_the_sums_of_its_chunks(n, d, chunk):
    """Two partial rows of d fp32 for each chunk, and a sorted list of keys and rows."""
    chunks = -(-n // chunk)
    assert E.eogp_embed_backward_workspace_size(n, 50257, d) >= chunks * (8 * d + 1) + 8 * n


def test_layer_norm_backward_asks_for_partial_sums_only():
    """Blocks that own an example write its gradients themselves: examples of few rows, or as many examples as
    blocks, need no room for partial sums, whatever their number."""
    size = E.eogp_layer_norm_backward_workspace_size
    for d, rows in ((768, 16), (768, 1), (5120, 4), (1024, 16), (16384, 4)):
        for code in (E.F32, E.BF16, E.F16):
            for groups in (1, 2, 131_072, 1 << 21):
                assert 0 < size(groups, rows, d, code) <= 256, (groups, rows, d)
    # 2 d fp32 for each block of a launch, of which there are at most twice 4 x 256 with partial sums
    for d in (768, 2048):
        for groups in (1, 128, 1023, 1024, 131_072):
            assert size(groups, 512, d, E.F32) <= 2048 * 2 * d * 4


@pytest.mark.parametrize("code", [E.F32, E.BF16, E.F16])
@pytest.mark.parametrize("d", [1, 5, 255, 768, 1025, 2047, 2049, 4097, 5120, 16384])
def test_layer_norm_backward_size_rises_with_groups_and_rows(d, code):
    size = E.eogp_layer_norm_backward_workspace_size
    for rows in (0, 1, 4, 5, 16, 17, 100, 512, 4096):
        assert_rising(lambda g: size(g, rows, d, code), range(1, 2200))
    for groups in (1, 2, 5, 128, 255, 256, 257, 600, 1023, 1024, 5000):
        assert_rising(lambda r: size(groups, r, d, code), range(0, 4200))


@pytest.mark.parametrize("pieces_of", [(E.F32, 4), (E.BF16, 8)])
def test_layer_norm_backward_size_holds_the_partial_sums(pieces_of):
    """2 d fp32 for each block, where a group has several: a group's blocks take four rows at a time (one, beyond
    256 pieces of 16 bytes), and 4 x 256 (256 beyond 512 pieces) fill the chip."""
    code, e = pieces_of
    for d in (64, 768, 1024, 1025, 2048, 2049, 4096, 4097, 16384):
        pieces = -(-d // e)
        per, fill = 4 if pieces <= 256 else 1, 1024 if pieces <= 512 else 256
        for groups in [*range(1, 300), 511, 512, 513, 1023, 1024, 4000]:
            for rows in (1, 5, 17, 40, 512, 3000):
                splits = min(-(-rows // per), -(-fill // groups)) if rows > 4 * per else 1
                need = groups * splits * 2 * d * 4 if splits > 1 else 0
                assert E.eogp_layer_norm_backward_workspace_size(groups, rows, d, code) >= need, (d, groups, rows)
