"""Which of its two ways a loss over a vocabulary goes, so that a test says which
one it is for: a change of the rule between them empties no test unnoticed."""
import paper_1601_04033_amd as fa


def way(m, d, V, dtype):
    """'direct' or 'tiles', by the workspace of a forward call: the direct way needs one for a mark a row and the
    statistics of its blocks alone, tiles for the rows that take part too."""
    def up(n, to):
        return -(-n // to) * to
    padded, groups = up(m, 16), up(V, 16) // 16
    tiles = padded // 16
    each = -(-groups // (256 // tiles)) if tiles < 256 else groups
    blocks = -(-groups // each)
    direct = up(4 * padded, 256) + up(8 * blocks * padded, 256) + up(4 * blocks * padded, 256)
    size = fa.client_vocab_workspace_bytes(m, d, V, dtype, backward=False)
    assert size == direct or size >= direct + 2 * up(m, 256) * up(d, 128), (m, d, V, dtype, size, direct)
    return "direct" if size == direct else "tiles"
