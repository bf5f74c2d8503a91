"""The limits of the paged cache's operators, at the last size that is taken and the first that is not.  A host-only
ctx answers a valid call with the status of one that is too large, so what is compared is the reason."""
import pytest

from paper_2606_31808_amd import lmop as L
from synth import SHAPES
from tests.test_operator_refusals import P, UNS, _call, _paged

VALID = "arguments are valid"
ONE = dict(batch_start=None, max_tokens=1)


class Wide:
    """Pages of 2^29 elements: 32,768 heads of 64 and 256 tokens."""
    n_layers, d_model, d_ff, vocab, group_size, rms_eps, rope_theta = 0, 64, 64, 2, 32, 1e-5, 1e4

    def __init__(self, heads):
        self.n_heads = self.n_kv_heads = heads
        self.head_dim = 64


def _why(ctx, name, **change):
    if name != "lmop_attend":
        change = {k: v for k, v in change.items() if k not in ("max_tokens", "workspace_bytes")}
    if name == "lmop_cache_append":
        change.pop("max_length", None)
    assert _call(ctx, name, _paged(ctx, name, **change)) == UNS
    return L._lib.lmop_last_error(ctx.ctx).decode()


@pytest.fixture(scope="module")
def ctx():
    c = L.Context(SHAPES["tiny"], device=-1)
    assert c.heads == (4, 4, 64)
    return c


ALL = ("lmop_cache_append", "lmop_attend", "lmop_select_blocks")


@pytest.mark.parametrize("name", ALL)
def test_a_valid_call_says_so(ctx, name):
    assert VALID in _why(ctx, name)


@pytest.mark.parametrize("name", ALL)
@pytest.mark.parametrize("taken,refused,reason", [
    # a sequence's table holds 2^30 keys
    (dict(batch_max_pages=2 ** 26, batch_ld_table=2 ** 26), dict(batch_max_pages=2 ** 26 + 1, batch_ld_table=2 ** 27),
     "pages of 16 tokens for a sequence"),
    # (tokens + 2 sequences) (4 + 2 * 4) heads: 2^24
    (dict(ONE, batch_n_tokens=466033, batch_n_seqs=466033), dict(ONE, batch_n_tokens=466034, batch_n_seqs=466034),
     "too many for one call"),
    (dict(batch_n_tokens=1398099, batch_n_seqs=1), dict(batch_n_tokens=1398100, batch_n_seqs=1), "too many for one call"),
    (dict(ONE, batch_n_tokens=466033, batch_n_seqs=466033),
     dict(ONE, batch_n_tokens=2 ** 31 - 1, batch_n_seqs=2 ** 31 - 1), "too many for one call")])
def test_batch_limits(ctx, name, taken, refused, reason):
    assert VALID in _why(ctx, name, **taken)
    assert reason in _why(ctx, name, **refused)


@pytest.mark.parametrize("name", ["lmop_cache_append", "lmop_attend"])
@pytest.mark.parametrize("taken,refused", [(dict(cache_page_stride=2 ** 32), dict(cache_page_stride=2 ** 32 + 16)),
                                           (dict(cache_page_stride=4112), dict(cache_page_stride=2 ** 40))])
def test_page_stride(ctx, name, taken, refused):
    assert VALID in _why(ctx, name, **taken)
    assert "pages of 4096 elements" in _why(ctx, name, **refused)


@pytest.mark.parametrize("name", ["lmop_cache_append", "lmop_attend"])
def test_page_elements(name):
    for heads, taken in ((32768, True), (32769, False)):
        wide = L.Context(Wide(heads), device=-1)
        page = heads * 64 * 256
        batch = dict(cache_page_size=256, cache_page_stride=page, batch_n_tokens=1, batch_n_seqs=1, max_tokens=1, ldq=heads * 64)
        more = dict(ldo=heads * 64) if name == "lmop_attend" else dict(ldk=heads * 64, ldv=heads * 64, ldqo=heads * 64)
        why = _why(wide, name, **batch, **more)
        assert (VALID in why) == taken
        assert taken or f"pages of {page} elements" in why


@pytest.mark.parametrize("taken,refused,reason", [
    (dict(prefix_length=2 ** 29, prefix=P), dict(prefix_length=2 ** 29 + 1, prefix=P), "a prefix of 536870913 keys"),
    (dict(prefix_length=2 ** 29, prefix=P), dict(prefix_length=2 ** 30, prefix=P), "a prefix of 1073741824 keys"),
    (dict(n_blocks=1024, blocks=P), dict(n_blocks=1025, blocks=P), "1025 blocks (at most 1024)"),
    # 65,535 splits of 512 pages
    (dict(ONE, batch_n_tokens=1, batch_n_seqs=1, batch_max_pages=65535 * 512, batch_ld_table=2 ** 26, max_length=65535 * 512 * 16),
     dict(ONE, batch_n_tokens=1, batch_n_seqs=1, batch_max_pages=65535 * 512 + 1, batch_ld_table=2 ** 26,
          max_length=65535 * 512 * 16 + 1), "too many for one call"),
    # 2^24 workgroups: sequences, 4 heads, 4096 splits
    (dict(ONE, batch_n_tokens=1023, batch_n_seqs=1023, cache_page_size=256, cache_page_stride=2 ** 16, batch_max_pages=2 ** 21,
          batch_ld_table=2 ** 21, max_length=2 ** 29, workspace_bytes=1 << 40),
     dict(ONE, batch_n_tokens=1024, batch_n_seqs=1024, cache_page_size=256, cache_page_stride=2 ** 16, batch_max_pages=2 ** 21,
          batch_ld_table=2 ** 21, max_length=2 ** 29, workspace_bytes=1 << 40), "too many for one call")])
def test_attend_limits(ctx, taken, refused, reason):
    assert VALID in _why(ctx, "lmop_attend", **taken)
    assert reason in _why(ctx, "lmop_attend", **refused)


@pytest.mark.parametrize("taken,refused,reason", [
    (dict(n_blocks=1024), dict(n_blocks=1025), "1025 blocks (at most 1024)"),
    (dict(max_length=16384 * 16), dict(max_length=16384 * 16 + 1), "at most 16384 pages of 16")])
def test_select_limits(ctx, taken, refused, reason):
    assert VALID in _why(ctx, "lmop_select_blocks", **taken)
    assert reason in _why(ctx, "lmop_select_blocks", **refused)
