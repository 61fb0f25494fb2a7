"""Sizes that reach every form of the projections: each kernel variant with whole K and with K over
workgroups, and where its copies have a way past the caches, that one too.

Tokens, features and columns lie off the tiles, K is several rings deep in every part.
"""
import ctypes

from paper_2609_38386_amd import dlfp as D

MOST = 32 << 20   # bytes of workspace that a form takes at most

# (tokens, features, columns, bytes of workspace)
SIZES = {
    D.LINEAR_W4: [
        (5, 1296, 2112, 0), (2, 22768, 5568, MOST), (3, 16, 14400, MOST), (2, 4720, 26816, MOST),
        (2, 12496, 64, MOST), (1, 4736, 14400, MOST), (1, 8272, 15552, MOST), (5, 16, 2112, MOST),
        (4, 10480, 12096, MOST), (5, 16, 16448, MOST), (3, 5456, 23744, MOST),
        (4, 4272, 2240, MOST), (4, 36432, 3520, MOST), (3, 4848, 14400, MOST),
        (4, 5072, 25280, MOST), (8, 13040, 2496, MOST), (8, 15984, 8000, MOST),
        (8, 1392, 23744, MOST), (8, 7696, 17600, MOST), (19, 2096, 2112, 0),
        (5, 592, 18496, MOST), (293, 16, 2112, MOST), (59, 16, 16448, MOST),
        (1373, 48, 2112, MOST), (225, 48, 16576, MOST), (2061, 48, 2112, MOST),
        (517, 48, 12736, MOST), (4103, 16, 2112, MOST), (531, 80, 11456, MOST),
        (4429, 48, 2112, MOST), (2075, 48, 7360, MOST), (4131, 48, 2112, 0),
        (2075, 48, 7744, MOST), (4187, 80, 2112, MOST), (19, 17520, 7232, MOST),
        (1431, 80, 9664, MOST), (5469, 144, 2112, MOST), (4115, 80, 6336, MOST),
        (6027, 528, 2112, MOST), (6175, 144, 7104, MOST), (6353, 272, 2112, MOST),
        (4135, 144, 6720, MOST), (7059, 816, 2112, MOST), (6297, 144, 8896, MOST),
        (7157, 1680, 2240, 1 << 20), (1351, 112, 17344, MOST), (5575, 112, 4288, MOST),
        (2183, 112, 12992, MOST), (1363, 16, 15808, MOST)],
    D.GATED_LINEAR_BF16: [
        (431, 16, 2112, 0), (16, 3184, 5440, MOST), (73, 16, 16960, MOST), (16, 1904, 8896, MOST),
        (9, 16, 2112, MOST), (8, 3920, 4288, MOST), (9, 16, 16960, MOST), (8, 656, 25664, MOST),
        (49, 720, 2496, MOST), (32, 3248, 5568, MOST), (1435, 16, 8512, MOST),
        (32, 912, 19008, MOST), (2747, 48, 2112, 0), (1369, 16, 2112, MOST),
        (4251, 80, 2112, MOST), (45, 8272, 2112, 0), (2461, 80, 6336, MOST),
        (64, 1232, 17600, MOST), (5733, 336, 2240, MOST), (69, 16464, 2112, 0),
        (5427, 80, 8512, MOST), (71, 8336, 6592, MOST), (4099, 48, 2112, MOST),
        (9, 8336, 2112, MOST), (449, 48, 17344, MOST), (32, 1392, 17088, MOST),
        (6759, 592, 2112, 0), (129, 16400, 2240, 1 << 20), (5719, 144, 2112, 0),
        (65, 8528, 2112, MOST), (5567, 80, 4672, MOST), (128, 1104, 18496, MOST),
        (6539, 272, 2112, 0), (15, 32816, 2112, MOST), (5519, 48, 28480, MOST),
        (45, 16432, 4416, MOST), (1033, 48, 12736, MOST), (2151, 16, 6336, 1 << 20)],
    D.GATED_LINEAR_W4: [
        (2, 4112, 2368, MOST), (2, 16784, 3776, MOST), (2, 688, 21184, MOST),
        (2, 2800, 22592, MOST), (9, 1360, 2112, 0), (4, 3568, 17984, MOST), (4, 304, 18496, MOST),
        (4, 2320, 30400, MOST), (8, 6800, 2240, MOST), (8, 28368, 2240, MOST),
        (8, 752, 20544, MOST), (8, 3088, 20928, MOST), (9, 16, 2112, MOST), (9, 16, 16448, MOST),
        (345, 16, 2112, MOST), (53, 16, 16448, MOST), (1101, 80, 2240, 1 << 20),
        (471, 48, 10304, MOST), (4119, 16, 2112, MOST), (1389, 16, 10432, MOST),
        (2773, 48, 2112, MOST), (857, 80, 7232, MOST), (2775, 48, 2624, MOST),
        (451, 48, 16960, MOST), (4111, 48, 2112, 0), (17, 8304, 7616, MOST),
        (1365, 48, 10176, MOST), (5477, 80, 2112, 0), (4247, 48, 6336, MOST),
        (5587, 272, 2112, 0), (6169, 80, 6592, MOST), (5777, 144, 2112, 0),
        (6215, 80, 4800, MOST), (7077, 400, 2112, 0), (6343, 80, 8640, MOST),
        (5163, 1168, 2112, MOST), (687, 112, 17344, MOST), (1409, 16, 9408, 1 << 20),
        (1061, 112, 12864, MOST)],
}

# Variants of few tokens, whose sums over workgroups are a kernel of their own, and those whose copies
# of weights may go past the caches.
FEW = {D.LINEAR_W4: range(13), D.GATED_LINEAR_BF16: range(3), D.GATED_LINEAR_W4: range(13)}
STREAMED = {D.LINEAR_W4: (0, 1, 2, 3, 4, 12), D.GATED_LINEAR_BF16: (0, 1, 2, 5, 6, 7, 8, 9, 10),
            D.GATED_LINEAR_W4: (1, 3, 4, 12)}


def forms_of(kind, m, n, k, room, form=None):
    """What a call of these sizes runs: (kind, variant, is K split, past the caches) of the first
    launch and, if K is split, (kind, of few tokens, splits) of the second.  None: refused."""
    form = form or D.dlfp_projection_form()
    if D.lib().dlfp_projection_form_of(kind, m, n, k, room, ctypes.byref(form)):
        return None
    split = form.splits > 1
    past = bool(form.past_caches) and form.variant in STREAMED[kind]
    first = (kind, form.variant, split, past)
    return {first, (kind, form.variant in FEW[kind], form.splits)} if split else {first}
