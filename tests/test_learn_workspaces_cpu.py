"""Workspaces of embedding, row norm and language-model loss (no GPU): one that is
large enough for some rows is large enough for fewer, and for fewer gradients."""
import pytest

import paper_2607_20357_amd as svl

WANT = [(False, False), (True, False), (False, True), (True, True)]


def _grows(size, rows):
    last = 0
    for n in rows:
        now = size(n)
        assert now >= last, (n, last, now)
        last = now


@pytest.mark.parametrize("d, vocab", [(64, 1), (256, 300), (256, 10240), (64, 16384), (1024, 20000), (4096, 32000),
                                      (64, 32768), (64, 32769), (1024, 65537), (4096, 151936), (64, 1 << 20)])
def test_loss_workspace_grows_with_the_rows(d, vocab):
    head = svl.make_lm_head(d, vocab)
    rows = list(range(0, 1400)) + list(range(1400, 9000, 127)) + [10000, 50000, 300000]
    for want in WANT:
        _grows(lambda n: svl.svl_lm_loss_workspace_bytes(head, n, *want), rows)
    for n in rows[::97]:
        most = svl.svl_lm_loss_workspace_bytes(head, n, True, True)
        assert all(svl.svl_lm_loss_workspace_bytes(head, n, *want) <= most for want in WANT)


def test_embedding_and_norm_workspaces_grow_with_the_rows():
    rows = list(range(0, 2100)) + list(range(2100, 40000, 331))
    for width, vocab in ((8, 1), (4096, 32000), (264, 255), (264, 256)):
        emb = svl.make_embedding(width, vocab)
        _grows(lambda n: svl.svl_embed_workspace_bytes(emb, n), rows)
    for width in (8, 1024, 1032, 16384):
        norm = svl.make_norm(width)
        _grows(lambda n: svl.svl_norm_workspace_bytes(norm, n), rows)
