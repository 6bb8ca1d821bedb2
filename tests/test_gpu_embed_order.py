"""The embedding gradient's order of sums, bit for bit: tokens sorted by id, added one by one within pieces of one size, the sums of a run
over several pieces by four chains of every fourth one."""
import numpy as np
import pytest
import torch

import paper_2410_20305_amd as ps

pytestmark = pytest.mark.gpu


def _chain(rows):
    s = np.zeros(rows.shape[1], dtype=np.float32)
    for r in rows:
        s = s + r
    return s


def _sums(ids, dX, vocab, piece):
    """What the calls promise, in fp32 on the host."""
    order = np.argsort(ids, kind="stable")
    out = np.zeros((vocab, dX.shape[1]), dtype=np.float32)
    for v in range(vocab):
        at = np.nonzero(ids[order] == v)[0]
        parts = [_chain(dX[order[at[at // piece == p]]]) for p in np.unique(at // piece)]
        if len(parts) == 1:
            out[v] = parts[0]
        elif parts:
            waves = [_chain(np.array(parts[w::4], dtype=np.float32).reshape(-1, dX.shape[1])) for w in range(4)]
            out[v] = ((waves[0] + waves[1]) + waves[2]) + waves[3]
    return out


def _got(ids, dX, vocab):
    return ps.psattn_embed_bwd(torch.from_numpy(ids.astype(np.int32)).cuda(), torch.from_numpy(dX).cuda(), vocab).cpu().numpy()


@pytest.mark.parametrize("T,vocab,counts", [
    (300, 40, None),                                   # runs of seven and eight, two of them across a cut
    (400, 3, [50, 170, 180]),                          # over two, six and seven pieces
    (1500, 4, [33, 700, 31, 736]),                     # over twenty and more
    (7000, 5, [1, 3000, 0, 3998, 1]),                  # sorted by digits instead of by counting; one id without a token
])
def test_in_pieces_and_their_joins(T, vocab, counts):
    rng = np.random.default_rng(T)
    ids = np.arange(T) % vocab if counts is None else rng.permutation(np.repeat(np.arange(vocab), counts))
    dX = (rng.standard_normal((T, 24)) * 10.0 ** rng.uniform(-3, 3, (T, 1))).astype(np.float32)
    assert np.array_equal(_got(ids, dX, vocab), _sums(ids, dX, vocab, 32))


def test_a_row_across_a_cut():
    """1 and then 2^-24 six times: one by one every 2^-24 is half a step of 1 and is dropped.  Id 24's tokens stand at sorted places
    188 .. 194, and the cut at 192 leaves three of the small ones to a sum of their own, which 1 then takes; id 7's are in one piece."""
    ids = np.arange(300) % 40
    dX = np.zeros((300, 8), dtype=np.float32)
    for v in (7, 24):
        mine = np.nonzero(ids == v)[0]
        dX[mine] = 2.0 ** -24
        dX[mine[0]] = 1.0
    got = _got(ids, dX, 40)
    assert np.all(got[7] == 1.0) and np.all(got[24] == np.float32(1.0) + np.float32(3 * 2.0 ** -24))
    # the same tokens of id 24 without others before them: in one piece
    keep = ids >= 24
    assert np.all(_got(ids[keep], dX[keep], 40)[24] == 1.0)
