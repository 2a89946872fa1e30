"""Products of few rows: the form that was measured to be faster is the one that is taken."""
from token_shapes import ask

# rows, results a row, bytes of an element; us without tiles and with them (MI355X), for sums over 4096 but where said
MEASURED = [
    (16, 4000, 2, 18.9, 26.8), (32, 4000, 2, 24.6, 28.7), (32, 8000, 2, 28.3, 33.1), (64, 1000, 2, 29.8, 24.1), (48, 1000, 2, 26.9, 22.8), (16, 32000, 2, 63.5, 70.8),
    (24, 12000, 2, 43.0, 33.5), (32, 32000, 2, 90.7, 70.9), (16, 128000, 2, 214.9, 185.9), (8, 128000, 2, 198.5, 183.7),
    (16, 200000, 2, 67.8, 49.6),                                   # sums over 512
    (64, 4000, 4, 61.8, 78.8), (64, 8000, 4, 65.1, 79.3), (24, 12000, 4, 74.6, 80.4), (48, 12000, 4, 108.3, 81.7), (32, 32000, 4, 172.4, 152.2), (16, 32000, 4, 128.6, 162.7),
    (32, 128000, 4, 622.1, 567.7), (16, 128000, 4, 451.0, 563.7),
    (24, 64000, 4, 58.8, 47.7),                                    # sums over 512
    (64, 4096, 1, 40.4, 46.4),                                     # sums over 14336
    (32, 4096, 1, 8.6, 11.6), (48, 8192, 1, 20.9, 15.7), (64, 8192, 1, 24.2, 16.3), (24, 8192, 1, 13.1, 14.6), (16, 14336, 1, 17.3, 19.4), (16, 28672, 1, 56.6, 61.0)]


def test_the_faster_form(tmp_path):
    taken = ask(tmp_path, [("few", m, n, esz) for m, n, esz, _, _ in MEASURED])
    for (m, n, esz, few, tiles), form in zip(MEASURED, taken):
        assert form == (few < tiles), (m, n, esz, few, tiles)
